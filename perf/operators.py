"""Cases of the operators of sequence policies (paper_1906_04585_b200.sequence): what is timed and compared.

Four operators, each as a user's program calls it and in a plain form of elementary torch operations in 32 bits:

  layer_norm   y = (s - mean s) / sqrt(var s + eps) * w + b over the columns of s = x (+ residual); with "train"
               also its backward pass (dx, dw, db; the residual path's gradient is added to dx)
  recurrence   h_t = a_t c_{t-1} + (1 - a_t) x_t with a_t = sigmoid(f_t), c_t = h_t or 0 where an episode (or packed
               document) ended at step t; with "train" also its backward pass (df, dx, dh0)
  ffn          y = (act(x Wg^T) * (x Wu^T)) Wd^T; with "train" also its backward pass (dx, dWg, dWu, dWd)
  sample       a token a row from temperature, top-k, top-p and min-p filtered logits and one given uniform number a
               row, with its log-probability

`own` chooses between the two.  Sizes are this repository's own (64 agents x 16 simulators = 1024 rows of acting, 512
hidden units, rollouts of 5 steps, 2..32 actions) or generic ones of sequence models.
"""
import math

import torch

own = False

EPS = 1e-5


def listed():
    return [
        # one acting step of 64 agents x 16 simulators through a pre-norm residual block of the framework's 512 units
        dict(name="ln act", op="layer_norm", rows=1024, cols=512, pad=0, dtype="bfloat16", wdtype="bfloat16", residual=True, train=False),
        # a training batch of a sequence model: eight sequences of 2048 tokens, weights kept in 32 bits
        dict(name="ln train", op="layer_norm", rows=16384, cols=2048, pad=0, dtype="bfloat16", wdtype="float32", residual=False, train=True),
        # a ragged batch of an odd width cut out of a wider buffer, in 32 bits, in the middle of a residual stream
        dict(name="ln train odd", op="layer_norm", rows=5121, cols=1001, pad=6, dtype="float32", wdtype="float32", residual=True, train=True),
        # one step of the memory of every simulator while acting
        dict(name="recurrence act", op="recurrence", steps=1, batch=1024, dim=512, dtype="bfloat16", done=0.01, train=False),
        # one long sequence read at once (a prompt, a recorded trajectory): little to run side by side but the time axis
        dict(name="recurrence long", op="recurrence", steps=65536, batch=1, dim=1024, dtype="bfloat16", done=0.0, train=False),
        # training on packed episodes
        dict(name="recurrence train", op="recurrence", steps=2048, batch=16, dim=2048, dtype="bfloat16", done=0.002, train=True),
        # decoding for a handful of sequences: the weights have to be read for a few rows
        dict(name="ffn decode", op="ffn", rows=7, dim=2048, hidden=8192, dtype="bfloat16", act="silu", train=False),
        # acting on a full batch of simulators, or reading a prompt
        dict(name="ffn act", op="ffn", rows=1024, dim=2048, hidden=8192, dtype="float16", act="gelu", train=False),
        # a training batch
        dict(name="ffn train", op="ffn", rows=8192, dim=2048, hidden=8192, dtype="bfloat16", act="silu", train=True),
        # the action draw of 64 agents x 16 simulators, nothing filtered
        dict(name="sample actions", op="sample", rows=1024, vocab=18, dtype="float32", filters="none"),
        # one token for each of 256 sequences, every request with settings of its own
        dict(name="sample batch", op="sample", rows=256, vocab=32768, dtype="bfloat16", filters="mixed"),
        # a large vocabulary in 32 bits
        dict(name="sample large", op="sample", rows=64, vocab=131072, dtype="float32", filters="mixed"),
    ]


def _log(rng, lo, hi):
    """A whole number in lo..hi, uniform on a logarithmic scale."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["layer_norm", "recurrence", "ffn", "sample"])
    if op == "layer_norm":
        cols = _log(rng, 32, 8192)
        residual = rng.random() < 0.5
        dtype = rng.choice(["bfloat16", "float16", "float32"])
        return dict(op=op, rows=_log(rng, 1, min(32768, (1 << 25) // cols)), cols=cols, pad=rng.choice([0, 0, 1, 8, 40]), dtype=dtype,
                    wdtype=dtype if residual else rng.choice([dtype, "float32"]), residual=residual, train=rng.random() < 0.6)
    if op == "recurrence":
        dim = _log(rng, 32, 4096)
        batch = _log(rng, 1, 1024)
        return dict(op=op, steps=_log(rng, 1, max(1, min(65536, (1 << 26) // (batch * dim)))), batch=batch, dim=dim,
                    dtype=rng.choice(["bfloat16", "float16", "float32"]), done=rng.choice([0.0, 0.002, 0.01, 0.2]), train=rng.random() < 0.6)
    if op == "ffn":
        dim, hidden = 8 * _log(rng, 8, 512), 8 * _log(rng, 16, 1024)
        return dict(op=op, rows=_log(rng, 1, max(1, min(8192, (1 << 37) // (dim * hidden)))), dim=dim, hidden=hidden,
                    dtype=rng.choice(["bfloat16", "float16"]), act=rng.choice(["silu", "gelu", "relu"]), train=rng.random() < 0.5)
    vocab = _log(rng, 2, 131072)
    return dict(op=op, rows=_log(rng, 1, min(1024, (1 << 23) // vocab)), vocab=vocab, dtype=rng.choice(["bfloat16", "float16", "float32"]),
                filters=rng.choice(["none", "mixed", "mixed"]))


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = getattr(torch, case["dtype"])

    def normal(*shape, std=1.0, mean=0.0, dtype=dt):
        return torch.randn(*shape, device="cuda", generator=gen).mul_(std).add_(mean).to(dtype)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=gen)

    s = dict(case)
    if case["op"] == "layer_norm":
        rows, cols, wdt = case["rows"], case["cols"], getattr(torch, case["wdtype"])
        # a residual stream: a mean that is not zero and a few columns much larger than the rest
        scale = torch.where(uniform(cols) < 0.01, 10.0, 1.0)

        def stream(std, mean):
            wide = torch.randn(rows, cols + case["pad"], device="cuda", generator=gen).mul_(std).add_(mean)
            wide[:, :cols] *= scale
            return wide.to(dt)[:, :cols]

        s["x"] = stream(1.0, 0.3)
        s["residual_in"] = stream(2.0, -0.1) if case["residual"] else None
        s["weight"] = normal(cols, std=0.2, mean=1.0, dtype=wdt)
        s["bias"] = normal(cols, std=0.1, dtype=wdt)
        s["dy"] = normal(rows, cols) if case["train"] else None
        s["dsum"] = normal(rows, cols) if case["train"] and case["residual"] else None
        s["y"] = torch.empty(rows, cols, device="cuda", dtype=dt)
        s["sum"] = torch.empty(rows, cols, device="cuda", dtype=dt) if case["residual"] else None
    elif case["op"] == "recurrence":
        T, B, D = case["steps"], case["batch"], case["dim"]
        # one projection of the layer's input gives both halves, as [time][sequence][2 x dim]
        both = torch.randn(T, B, 2 * D, device="cuda", generator=gen)
        both[..., :D].mul_(1.5).add_(2.0)   # gates that mostly remember: a memory of some ten steps, up to some hundred
        both = both.to(dt)
        s["f"], s["x"] = both[..., :D], both[..., D:]
        s["h0"] = normal(B, D, dtype=torch.float32, std=0.5)
        s["done_in"] = (uniform(T, B) < case["done"]).to(torch.uint8) if case["done"] else None
        s["dh"] = normal(T, B, D) if case["train"] else None
        s["dh_last"] = normal(B, D, dtype=torch.float32) if case["train"] else None
        s["h"] = torch.empty(T, B, D, device="cuda", dtype=dt)
        s["h_last"] = torch.empty(B, D, device="cuda")
    elif case["op"] == "ffn":
        M, D, F = case["rows"], case["dim"], case["hidden"]
        s["x"] = normal(M, D)
        s["w_gate"] = normal(F, D, std=D ** -0.5)
        s["w_up"] = normal(F, D, std=D ** -0.5)
        s["w_down"] = normal(D, F, std=F ** -0.5)
        s["dy"] = normal(M, D) if case["train"] else None
        s["y"] = torch.empty(M, D, device="cuda", dtype=dt)
    else:
        R, V = case["rows"], case["vocab"]
        s["logits"] = normal(R, V, std=2.5)
        if V <= 32:     # actions: some are not allowed in a state, the first always is
            s["logits"][:, 1:][uniform(R, V - 1) < 0.2] = -math.inf
        s["uniforms"] = uniform(R)
        if case["filters"] == "mixed":
            # each request has its own settings; some switch a filter off, some decode greedily
            kind = torch.randint(0, 8, (R,), device="cuda", generator=gen)
            s["temperature"] = torch.where(kind == 0, 0.0, 0.6 + 0.6 * uniform(R))
            s["top_k"] = torch.where(kind % 2 == 0, torch.randint(1, 201, (R,), device="cuda", generator=gen), 0).to(torch.int32)
            s["top_p"] = torch.where(kind < 5, 0.8 + 0.18 * uniform(R), 1.0)
            s["min_p"] = torch.where(kind % 3 == 0, 0.02 + 0.08 * uniform(R), 0.0)
        else:
            s["temperature"] = s["top_k"] = s["top_p"] = s["min_p"] = None
        s["tokens"] = torch.empty(R, device="cuda", dtype=torch.int32)
        s["logprobs"] = torch.empty(R, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _OWN[state["op"]](state)
    return _PLAIN[state["op"]](state)


def _own_layer_norm(s):
    from paper_1906_04585_b200 import sequence as S
    y, total, mean, rstd = S.layer_norm(s["x"], s["weight"], s["bias"], EPS, residual=s["residual_in"], out=s["y"], sum_out=s["sum"])
    out = {"y": y}
    if s["residual"]:
        out["sum"] = total
    if s["train"]:
        out["dx"], out["dw"], out["db"] = S.layer_norm_backward(s["dy"], total if s["residual"] else s["x"], mean, rstd, s["weight"],
                                                                dsum=s["dsum"])
    return out


def _own_recurrence(s):
    from paper_1906_04585_b200 import sequence as S
    h, last, states = S.gated_recurrence(s["f"], s["x"], s["h0"], done=s["done_in"], out=s["h"], h_last=s["h_last"], save=s["train"])
    out = {"h": h, "h_last": last}
    if s["train"]:
        out["df"], out["dx"], out["dh0"] = S.gated_recurrence_backward(s["dh"], s["f"], s["x"], states, done=s["done_in"], dh_last=s["dh_last"])
    return out


def _own_ffn(s):
    from paper_1906_04585_b200 import sequence as S
    y, saved = S.gated_ffn(s["x"], s["w_gate"], s["w_up"], s["w_down"], s["act"], out=s["y"], save=s["train"])
    out = {"y": y}
    if s["train"]:
        out["dx"], out["dw_gate"], out["dw_up"], out["dw_down"] = S.gated_ffn_backward(s["dy"], s["x"], s["w_gate"], s["w_up"], s["w_down"],
                                                                                       saved, s["act"])
    return out


def _own_sample(s):
    from paper_1906_04585_b200 import sequence as S
    tokens, logprobs = S.sample(s["logits"], s["uniforms"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], out=s["tokens"],
                                logprobs=s["logprobs"])
    return {"tokens": tokens, "logprobs": logprobs}


_OWN = {"layer_norm": _own_layer_norm, "recurrence": _own_recurrence, "ffn": _own_ffn, "sample": _own_sample}


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_layer_norm(s):
    dt, wdt = s["x"].dtype, s["weight"].dtype
    x, w = s["x"].float(), s["weight"].float()
    if s["residual"]:
        x = x + s["residual_in"].float()
    centred = x - x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((centred * centred).mean(1, keepdim=True) + EPS)
    xhat = centred * rstd
    out = {"y": (xhat * w + s["bias"].float()).to(dt)}
    if s["residual"]:
        out["sum"] = x.to(dt)
    if s["train"]:
        dy = s["dy"].float()
        wdy = dy * w
        dx = rstd * (wdy - wdy.mean(1, keepdim=True) - xhat * (wdy * xhat).mean(1, keepdim=True))
        if s["residual"]:
            dx = dx + s["dsum"].float()
        out["dx"], out["dw"], out["db"] = dx.to(dt), (dy * xhat).sum(0).to(wdt), dy.sum(0).to(wdt)
    return out


def _scan(a, b):
    """v_t = a_t v_{t-1} + b_t along the first axis, v before it being 0, by doubling: after a step of width w every
    entry stands for the 2w steps that end with it, so log2(length) steps do.  (A torch program without a kernel of
    its own has no shorter way: one operation a time step would be tens of thousands.)"""
    width = 1
    while width < a.shape[0]:
        b = torch.cat([b[:width], b[width:] + a[width:] * b[:-width]])
        a = torch.cat([a[:width], a[width:] * a[:-width]])
        width *= 2
    return b


def _plain_recurrence(s):
    dt = s["x"].dtype
    f, x, h0 = s["f"].float(), s["x"].float(), s["h0"]
    T = f.shape[0]
    a, b = 1.0 / (1.0 + torch.exp(-f)), 1.0 / (1.0 + torch.exp(f))
    keep = torch.ones(T, f.shape[1], 1, device=f.device) if s["done_in"] is None else (s["done_in"] == 0).float().unsqueeze(-1)
    carry = torch.cat([torch.ones_like(keep[:1]), keep[:-1]]) * a    # what step t takes over from step t - 1
    start = b * x
    start[0] += a[0] * h0
    h = _scan(carry, start)
    out = {"h": h.to(dt), "h_last": h[-1] * keep[-1]}
    if s["train"]:
        dh = s["dh"].float()
        dh[-1] += s["dh_last"] * keep[-1]
        # g_t = dh_t + carry_{t+1} g_{t+1}: the same scan from the other end
        back = torch.cat([carry[1:], torch.zeros_like(carry[:1])])
        g = _scan(back.flip(0), dh.flip(0)).flip(0)
        before = torch.cat([h0.unsqueeze(0), h[:-1] * keep[:-1]])
        out["df"], out["dx"], out["dh0"] = (g * (before - x) * a * b).to(dt), (g * b).to(dt), g[0] * a[0]
    return out


def _act(g, act):
    if act == "silu":
        return g / (1.0 + torch.exp(-g))
    if act == "gelu":
        return 0.5 * g * (1.0 + torch.erf(g * 0.7071067811865476))
    return g * (g > 0)


def _act_slope(g, act):
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return p * (1.0 + g * (1.0 - p))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(g * 0.7071067811865476)) + g * torch.exp(-0.5 * g * g) * 0.3989422804014327
    return (g > 0).float()


def _plain_ffn(s):
    dt, act = s["x"].dtype, s["act"]
    x, wg, wu, wd = s["x"].float(), s["w_gate"].float(), s["w_up"].float(), s["w_down"].float()
    g, u = x @ wg.T, x @ wu.T
    v = _act(g, act)
    h = v * u
    out = {"y": (h @ wd.T).to(dt)}
    if s["train"]:
        dy = s["dy"].float()
        dh = dy @ wd
        dg, du = dh * u * _act_slope(g, act), dh * v
        out["dx"] = (dg @ wg + du @ wu).to(dt)
        out["dw_gate"], out["dw_up"], out["dw_down"] = (dg.T @ x).to(dt), (du.T @ x).to(dt), (dy.T @ h).to(dt)
    return out


def _plain_sample(s):
    # The draw is a whole number, so the running sums that decide it are kept in 64 bits; the weights are 32-bit.
    logits = s["logits"].float()
    R, V = logits.shape
    logits = torch.where(torch.isnan(logits), -math.inf, logits)
    order = torch.sort(logits, dim=1, descending=True, stable=True)   # ties: lowest index first
    top = order.values[:, :1]
    t = torch.ones(R, 1, device=logits.device) if s["temperature"] is None else s["temperature"].unsqueeze(1)
    greedy = t <= 0
    # a logit equal to the largest weighs 1 whatever it is (infinite, or the type's lowest value in every place)
    w = torch.where(order.values == top, 1.0, torch.exp((order.values - top) / torch.where(greedy, 1.0, t)))
    rank = torch.arange(V, device=logits.device).unsqueeze(0)
    keep = torch.where(greedy, rank < 1, top > -math.inf)
    if s["top_k"] is not None:
        k = s["top_k"].unsqueeze(1)
        keep = keep & ((k <= 0) | (rank < k))
    if s["top_p"] is not None:
        p = s["top_p"].unsqueeze(1)
        mass = torch.where(keep, w, 0.0).double()
        before = torch.cumsum(mass, 1) - mass
        keep = keep & ((p >= 1.0) | (before < p.double() * mass.sum(1, keepdim=True)) | (rank < 1))
    if s["min_p"] is not None:
        keep = keep & (w >= s["min_p"].unsqueeze(1))
    kept = torch.zeros(R, V, device=logits.device).scatter_(1, order.indices, torch.where(keep, w, 0.0))   # back in the order of the index
    run_sum = torch.cumsum(kept.double(), 1)
    total = run_sum[:, -1:]
    drawn = (run_sum > s["uniforms"].double().unsqueeze(1) * total) & (kept > 0)
    token = torch.argmax(drawn.to(torch.int8), 1)
    weight = kept.gather(1, token.unsqueeze(1))
    logprob = torch.log(weight.double() / total).float()[:, 0]
    empty = top[:, 0] == -math.inf
    return {"tokens": torch.where(empty, -1, token).to(torch.int32), "logprobs": torch.where(empty, -math.inf, logprob)}


_PLAIN = {"layer_norm": _plain_layer_norm, "recurrence": _plain_recurrence, "ffn": _plain_ffn, "sample": _plain_sample}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    e = 4 if case["dtype"] == "float32" else 2
    if case["op"] == "layer_norm":
        n, c = case["rows"] * case["cols"], case["cols"]
        we = 4 if case["wdtype"] == "float32" else 2
        moved, ops = n * e * (4 if case["residual"] else 2) + 2 * c * we, 8 * n
        if case["train"]:   # dy (and the residual path's gradient) read, the normalised input read again, dx written
            moved, ops = moved + n * e * (4 if case["residual"] else 3) + 3 * c * we, ops + 14 * n
        return {"bytes": moved, "flops": ops}
    if case["op"] == "recurrence":
        rows, n = case["steps"] * case["batch"], case["steps"] * case["batch"] * case["dim"]
        state, flags = 4 * case["batch"] * case["dim"], rows if case["done"] else 0
        moved, ops = 3 * n * e + 2 * state + flags, 8 * n
        if case["train"]:
            moved, ops = moved + 5 * n * e + 2 * state + flags, ops + 20 * n
        return {"bytes": moved, "flops": ops}
    if case["op"] == "ffn":
        m, d, f = case["rows"], case["dim"], case["hidden"]
        moved, ops = 2 * m * d * e + 3 * d * f * e, 6 * m * d * f
        if case["train"]:
            moved, ops = moved + 2 * m * d * e + 3 * d * f * e, ops + 12 * m * d * f
        return {"bytes": moved, "flops": ops}
    n = case["rows"] * case["vocab"]
    return {"bytes": n * e + case["rows"] * (28 if case["filters"] == "mixed" else 12), "flops": 6 * n}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"layer_norm": _exact_layer_norm, "recurrence": _exact_recurrence, "ffn": _exact_ffn, "sample": _exact_sample}[case["op"]](s)


def _exact_layer_norm(s):
    v = s["x"].double() if not s["residual"] else s["x"].double() + s["residual_in"].double()
    n = v.shape[1]
    mean = v.sum(1, keepdim=True) / n
    var = (v - mean).pow(2).sum(1, keepdim=True) / n
    z = (v - mean) / (var + EPS).sqrt()
    out = {"y": z * s["weight"].double() + s["bias"].double()}
    if s["residual"]:
        out["sum"] = v
    if s["train"]:
        dy = s["dy"].double()
        dz = dy * s["weight"].double()
        # through the variance and through the mean, term by term
        dvar = (dz * (v - mean)).sum(1, keepdim=True) * -0.5 * (var + EPS).pow(-1.5)
        dmean = -dz.sum(1, keepdim=True) / (var + EPS).sqrt()
        dx = dz / (var + EPS).sqrt() + dvar * 2.0 * (v - mean) / n + dmean / n
        out["dx"] = dx + s["dsum"].double() if s["residual"] else dx
        out["dw"], out["db"] = torch.einsum("rc,rc->c", dy, z), torch.einsum("rc->c", dy)
    return out


def _exact_recurrence(s):
    """Step by step, many pieces of the time axis side by side: inside a piece first with nothing carried in, then the
    pieces are joined one after another."""
    f, x = s["f"].double(), s["x"].double()
    T, B, D = f.shape
    piece = max(1, math.isqrt(T))
    pieces = -(-T // piece)
    length = pieces * piece
    keep = torch.ones(T, B, device=f.device, dtype=torch.float64) if s["done_in"] is None else 1.0 - s["done_in"].double()

    def steps(gain, add, first):
        """v_t = gain_t v_{t-1} + add_t, v_{-1} = first."""
        g = torch.ones(length, B, D, device=f.device, dtype=torch.float64)
        v = torch.zeros_like(g)
        g[:T], v[:T] = gain, add
        g, v = g.view(pieces, piece, B, D), v.view(pieces, piece, B, D)
        for i in range(1, piece):
            v[:, i] += g[:, i] * v[:, i - 1]
            g[:, i] *= g[:, i - 1]
        for p in range(pieces):
            v[p] += g[p] * first
            first = v[p, -1].clone()
        return v.view(length, B, D)[:T]

    a = torch.sigmoid(f)
    into = a.clone()                       # what step t takes over from h_{t-1}
    into[1:] *= keep[:-1].unsqueeze(-1)
    h = steps(into, torch.sigmoid(-f) * x, s["h0"].double())
    out = {"h": h, "h_last": h[-1] * keep[-1].unsqueeze(-1)}
    if s["train"]:
        dh = s["dh"].double()
        dh[-1] += s["dh_last"].double() * keep[-1].unsqueeze(-1)
        over = torch.zeros_like(into)
        over[:-1] = into[1:]
        g = steps(over.flip(0), dh.flip(0), torch.zeros(B, D, device=f.device, dtype=torch.float64)).flip(0)
        before = torch.empty_like(h)
        before[0], before[1:] = s["h0"].double(), h[:-1] * keep[:-1].unsqueeze(-1)
        out["df"], out["dx"], out["dh0"] = g * (before - x) * a * torch.sigmoid(-f), g * torch.sigmoid(-f), g[0] * a[0]
    return out


def _exact_ffn(s):
    def act(g):
        if s["act"] == "silu":
            return g * torch.sigmoid(g)
        if s["act"] == "gelu":
            return g * 0.5 * torch.special.erfc(-g / math.sqrt(2.0))
        return torch.clamp(g, min=0.0)

    def slope(g):
        if s["act"] == "silu":
            return torch.sigmoid(g) + g * torch.sigmoid(g) * torch.sigmoid(-g)
        if s["act"] == "gelu":
            return 0.5 * torch.special.erfc(-g / math.sqrt(2.0)) + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        return torch.where(g > 0, 1.0, 0.0).double()

    x, wg, wu, wd = (s[k].double() for k in ("x", "w_gate", "w_up", "w_down"))
    g, u = torch.einsum("md,fd->mf", x, wg), torch.einsum("md,fd->mf", x, wu)
    h = act(g) * u
    out = {"y": torch.einsum("mf,df->md", h, wd)}
    if s["train"]:
        dy = s["dy"].double()
        dh = torch.einsum("md,df->mf", dy, wd)
        dg, du = dh * u * slope(g), dh * act(g)
        out["dx"] = torch.einsum("mf,fd->md", dg, wg) + torch.einsum("mf,fd->md", du, wu)
        out["dw_gate"], out["dw_up"] = torch.einsum("mf,md->fd", dg, x), torch.einsum("mf,md->fd", du, x)
        out["dw_down"] = torch.einsum("md,mf->df", dy, h)
    return out


def _exact_sample(s):
    """Row by row on the definition: rank, cut, cut, cut, draw."""
    logits = s["logits"].double()
    R, V = logits.shape
    tokens = torch.empty(R, dtype=torch.int32, device=logits.device)
    logprobs = torch.empty(R, dtype=torch.float64, device=logits.device)
    t, k, p, m = ([None] * R if s[n] is None else s[n].tolist() for n in ("temperature", "top_k", "top_p", "min_p"))
    uniforms = s["uniforms"].tolist()
    for r in range(R):
        row = logits[r]
        if t[r] is not None and t[r] <= 0:
            tokens[r], logprobs[r] = torch.nonzero(row == row.max())[0, 0], 0.0
            continue
        w = torch.exp((row - row.max()) / (1.0 if t[r] is None else t[r]))
        ranked = torch.argsort(row, descending=True, stable=True)
        if k[r]:
            ranked = ranked[:k[r]]
        if p[r] is not None and p[r] < 1.0:
            mass = w[ranked]
            ranked = ranked[:max(1, int((mass.cumsum(0) - mass < p[r] * mass.sum()).sum()))]
        if m[r]:
            ranked = ranked[w[ranked] >= m[r]]
        kept = torch.sort(ranked).values
        cdf = w[kept].cumsum(0)
        at = min(int((cdf <= uniforms[r] * cdf[-1]).sum()), len(kept) - 1)
        tokens[r], logprobs[r] = kept[at], torch.log(w[kept[at]] / cdf[-1])
    return {"tokens": tokens, "logprobs": logprobs}
