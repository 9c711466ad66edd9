"""Cases of the attention-memory operators and of the logit adjustments (paper_1906_04585_b200.sequence): what is timed and
compared.

Three operators, each as a user's program calls it and in a plain form of elementary torch operations in 32 bits:

  attention  a matrix memory a head: S_t = g C_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t, C_t = S_t or 0 where an episode (or
             packed document) ended at step t, g = exp(log_decay) of the head; from s0 to s_last; with "train" also its
             backward pass (dq, dk, dv, ds0)
  qk         queries and keys normed by head, x / sqrt(mean x^2 + eps) * w, and turned by position: pair i of the first
             2 x pairs entries by the angle position * inv_freq_i; with "train" also its backward pass (dq, dk, dwq, dwk)
  adjust     logits before a draw: penalties of the tokens in each row's history (repetition, frequency, presence), biases
             of listed tokens, a bit mask of what is allowed

`own` chooses between the two.  Sizes are this repository's own (64 agents x 16 simulators = 1024 rows of acting, 512 units as
8 heads of 64, rollouts of 5 steps, 2..32 actions) or generic ones of sequence models.
"""
import math

import torch

own = False

EPS = 1e-6


def listed():
    return [
        # one acting step of 64 agents x 16 simulators: every simulator's memory is read and written once
        dict(name="attention act", op="attention", steps=1, batch=1024, heads=8, dk=64, dv=64, dtype="bfloat16", layout="time", done=0.01, train=False),
        # one token for a handful of sequences, where latency counts
        dict(name="attention decode", op="attention", steps=1, batch=7, heads=16, dk=128, dv=128, dtype="float16", layout="time", done=0.0, train=False),
        # learning from a rollout of five steps
        dict(name="attention rollout", op="attention", steps=5, batch=1024, heads=8, dk=64, dv=64, dtype="bfloat16", layout="time", done=0.01, train=True),
        # one long sequence read at once (a prompt, a recorded trajectory): little to run side by side but the time axis
        dict(name="attention prompt", op="attention", steps=16384, batch=1, heads=16, dk=128, dv=128, dtype="bfloat16", layout="time", done=0.0, train=False),
        # training on packed episodes
        dict(name="attention train", op="attention", steps=2048, batch=8, heads=16, dk=128, dv=128, dtype="bfloat16", layout="sequence", done=0.002, train=True),
        # a ragged batch with heads of two odd sizes, in 32 bits
        dict(name="attention train odd", op="attention", steps=777, batch=3, heads=5, dk=41, dv=72, dtype="float32", layout="sequence", done=0.01, train=True),
        # the queries and keys of one acting step
        dict(name="qk act", op="qk", tokens=1024, q_heads=8, k_heads=8, dim=64, pairs=32, interleaved=False, dtype="bfloat16", wdtype="bfloat16", far=4096, train=False),
        # a training batch, keys shared by groups of four heads
        dict(name="qk train", op="qk", tokens=16384, q_heads=16, k_heads=4, dim=128, pairs=64, interleaved=False, dtype="bfloat16", wdtype="float32", far=2048, train=True),
        # heads of an odd size turned in part, neighbours paired, far into a sequence, in 32 bits
        dict(name="qk train odd", op="qk", tokens=5121, q_heads=5, k_heads=3, dim=75, pairs=20, interleaved=True, dtype="float32", wdtype="float32", far=1 << 20, train=True),
        # the action masks of 64 agents x 16 simulators
        dict(name="adjust actions", op="adjust", rows=1024, vocab=18, dtype="float32", history=0, biases=0, mask=True),
        # one token for each of 256 sequences, every request with settings of its own
        dict(name="adjust batch", op="adjust", rows=256, vocab=32768, dtype="bfloat16", history=2048, biases=64, mask=True),
        # a large vocabulary in 32 bits, long histories
        dict(name="adjust large", op="adjust", rows=64, vocab=131072, dtype="float32", history=8192, biases=300, mask=True),
    ]


def _log(rng, lo, hi):
    """A whole number in lo..hi, uniform on a logarithmic scale."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "qk", "adjust"])
    if op == "attention":
        dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
        dk, dv = (rng.randint(8, 128), rng.randint(8, 128)) if dtype == "float32" else (8 * rng.randint(2, 16), 8 * rng.randint(2, 16))
        heads = _log(rng, 1, 32)
        batch = _log(rng, 1, max(1, 2048 // heads))
        return dict(op=op, steps=_log(rng, 1, max(1, min(16384, (1 << 18) // (batch * heads)))), batch=batch, heads=heads, dk=dk, dv=dv, dtype=dtype,
                    layout=rng.choice(["time", "sequence"]), done=rng.choice([0.0, 0.002, 0.01, 0.2]), train=rng.random() < 0.5)
    if op == "qk":
        dtype = rng.choice(["bfloat16", "float16", "float32"])
        dim = rng.choice([64, 128, 256, 8 * rng.randint(2, 32), rng.randint(16, 256)])
        q_heads = _log(rng, 1, 32)
        k_heads = max(1, q_heads // rng.choice([1, 2, 4, 8]))
        return dict(op=op, tokens=_log(rng, 1, max(1, min(32768, (1 << 25) // (dim * (q_heads + k_heads))))), q_heads=q_heads, k_heads=k_heads, dim=dim,
                    pairs=dim // 2 if rng.random() < 0.7 else rng.randint(1, dim // 2), interleaved=rng.random() < 0.4, dtype=dtype,
                    wdtype=rng.choice([dtype, "float32"]), far=_log(rng, 1024, 1 << 20), train=rng.random() < 0.5)
    vocab = _log(rng, 2, 131072)
    history, biases = rng.choice([0, _log(rng, 1, 8192)]), rng.choice([0, _log(rng, 1, 300)])
    return dict(op=op, rows=_log(rng, 1, min(1024, (1 << 23) // vocab)), vocab=vocab, dtype=rng.choice(["bfloat16", "float16", "float32"]),
                history=history, biases=biases, mask=rng.random() < 0.6 or history + biases == 0)


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = getattr(torch, case["dtype"])

    def normal(*shape, std=1.0, mean=0.0, dtype=dt):
        return torch.randn(*shape, device="cuda", generator=gen).mul_(std).add_(mean).to(dtype)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=gen)

    def below(n, *shape):
        return torch.randint(0, n, shape, device="cuda", generator=gen)

    s = dict(case)
    if case["op"] == "attention":
        T, N, H, dk, dv = (case[n] for n in ("steps", "batch", "heads", "dk", "dv"))

        def steps(width):
            if case["layout"] == "sequence":
                return normal(N, T, width).transpose(0, 1)
            return normal(T, N, width)

        # one projection of the layer's input gives all three
        qkv = steps(H * (2 * dk + dv))
        s["q"], s["k"] = qkv[..., :H * dk].unflatten(2, (H, dk)), qkv[..., H * dk:2 * H * dk].unflatten(2, (H, dk))
        s["v"] = qkv[..., 2 * H * dk:].unflatten(2, (H, dv))
        s["scale"] = dk ** -0.5
        # heads that remember for 4 to 256 steps
        s["log_decay"] = torch.log1p(-torch.exp2(-torch.linspace(2.0, 8.0, H, device="cuda", dtype=torch.float64))).float()
        s["s0"] = normal(N, H, dk, dv, dtype=torch.float32)
        s["done_in"] = (uniform(T, N) < case["done"]).to(torch.uint8) if case["done"] else None
        s["do"] = steps(H * dv).unflatten(2, (H, dv)) if case["train"] else None
        s["ds_last"] = normal(N, H, dk, dv, dtype=torch.float32) if case["train"] else None
        s["o"] = torch.empty(T, N, H, dv, device="cuda", dtype=dt)
        s["s_last"] = torch.empty(N, H, dk, dv, device="cuda")
    elif case["op"] == "qk":
        n, hq, hk, d, wdt = case["tokens"], case["q_heads"], case["k_heads"], case["dim"], getattr(torch, case["wdtype"])
        # the projection's output with the values behind the queries and keys
        qkv = normal(n, (hq + 2 * hk) * d, std=1.5)
        s["q"], s["k"] = qkv[:, :hq * d].unflatten(1, (hq, d)), qkv[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d))
        s["wq"], s["wk"] = normal(d, std=0.2, mean=1.0, dtype=wdt), normal(d, std=0.2, mean=1.0, dtype=wdt)
        s["positions"] = below(case["far"], n).to(torch.int32)
        s["inv_freq"] = torch.pow(10000.0, -torch.arange(case["pairs"], device="cuda", dtype=torch.float64) / case["pairs"]).float()
        s["dq"], s["dk"] = (normal(n, hq, d), normal(n, hk, d)) if case["train"] else (None, None)
        s["q_out"], s["k_out"] = torch.empty(n, hq, d, device="cuda", dtype=dt), torch.empty(n, hk, d, device="cuda", dtype=dt)
    else:
        R, V, W, B = case["rows"], case["vocab"], case["history"], case["biases"]
        s["logits"] = normal(R, V, std=2.5)
        s["history_in"] = s["lengths"] = s["repetition"] = s["frequency"] = s["presence"] = None
        if W:
            # few tokens make up most of a text; requests are in the middle of theirs, some have switched a penalty off
            s["history_in"] = (V * uniform(R, W).pow(4)).to(torch.int32).clamp_(max=V - 1)
            s["lengths"] = below(W + 1, R).to(torch.int32)
            kind = below(4, R)
            s["repetition"] = torch.where(kind == 0, 1.0, 1.0 + 0.3 * uniform(R))
            s["frequency"] = torch.where(kind == 1, 0.0, 0.5 * uniform(R))
            s["presence"] = torch.where(kind == 2, 0.0, 0.5 * uniform(R))
        s["bias_ids"] = s["bias_values"] = None
        if B:     # shorter lists are filled up with -1
            s["bias_ids"] = torch.where(uniform(R, B) < 0.2, -1, below(V, R, B)).to(torch.int32)
            s["bias_values"] = normal(R, B, std=3.0, dtype=torch.float32)
        # a grammar allows about half of the vocabulary
        s["mask_in"] = torch.randint(-(1 << 31), 1 << 31, (R, (V + 31) // 32), device="cuda", generator=gen).to(torch.int32) if case["mask"] else None
        s["out"] = torch.empty(R, V, device="cuda", dtype=dt)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _OWN[state["op"]](state)
    return _PLAIN[state["op"]](state)


def _own_attention(s):
    from paper_1906_04585_b200 import sequence as S
    o, last = S.linear_attention(s["q"], s["k"], s["v"], s["log_decay"], s["s0"], done=s["done_in"], scale=s["scale"], out=s["o"], s_last=s["s_last"])
    out = {"o": o, "s_last": last}
    if s["train"]:
        out["dq"], out["dk"], out["dv"], out["ds0"] = S.linear_attention_backward(s["do"], s["q"], s["k"], s["v"], s["log_decay"], s["s0"],
                                                                                  done=s["done_in"], scale=s["scale"], ds_last=s["ds_last"])
    return out


def _own_qk(s):
    from paper_1906_04585_b200 import sequence as S
    q, k = S.qk_norm_rotary(s["q"], s["k"], s["positions"], s["inv_freq"], s["wq"], s["wk"], EPS, interleaved=s["interleaved"], q_out=s["q_out"], k_out=s["k_out"])
    out = {"q": q, "k": k}
    if s["train"]:
        out["dq"], out["dk"], out["dwq"], out["dwk"] = S.qk_norm_rotary_backward(s["dq"], s["dk"], s["q"], s["k"], s["positions"], s["inv_freq"],
                                                                                 s["wq"], s["wk"], EPS, interleaved=s["interleaved"])
    return out


def _own_adjust(s):
    from paper_1906_04585_b200 import sequence as S
    return S.adjust_logits(s["logits"], history=s["history_in"], lengths=s["lengths"], repetition=s["repetition"], frequency=s["frequency"],
                           presence=s["presence"], bias_ids=s["bias_ids"], bias_values=s["bias_values"], mask=s["mask_in"], out=s["out"])


_OWN = {"attention": _own_attention, "qk": _own_qk, "adjust": _own_adjust}


# ------------------------------------------------------------------------------------------------ plain forms
CHUNK = 64


def _memory(q, k, v, log_decay, cut, first, entry):
    """o_i = sum over j <= i of g^(i-j) (q_i . k_j) v_j + g^(i+entry) q_i first, and the sum of the same kind that is left
    after the last step; no term crosses a cut, which stands before the step that it is set for.  Step by step this would be
    an operation a step; by chunks it is a few products: within a chunk, and from the chunks before it."""
    T, N, H, dk = q.shape
    dv = v.shape[-1]
    chunk = min(CHUNK, T)
    n = -(-T // chunk)
    pad = n * chunk - T

    def chunks(x):    # [T, N, H, d] -> [N, H, n, chunk, d]
        x = torch.cat([x, x.new_zeros(pad, N, H, x.shape[-1])])
        return x.view(n, chunk, N, H, -1).permute(2, 3, 0, 1, 4)

    q, k, v = chunks(q), chunks(k), chunks(v)
    run = torch.cumsum(torch.cat([cut, cut.new_zeros(pad, N)]).to(torch.int32), 0).view(n, chunk, N).permute(2, 0, 1).unsqueeze(1)    # [N, 1, n, chunk]
    at = torch.arange(chunk, device=q.device)
    end = min(chunk, T) - 1

    def power(e):     # g^e for whole numbers e >= 0, [H, *e.shape]
        e = e.float().unsqueeze(0)
        return torch.where(e > 0, torch.exp(log_decay.view(-1, *[1] * (e.dim() - 1)) * e), 1.0)

    gap = at.view(-1, 1) - at.view(1, -1)
    link = torch.where((gap >= 0) & (run.unsqueeze(-1) == run.unsqueeze(-2)), power(gap.clamp(min=0)).unsqueeze(1), 0.0)
    o = ((q @ k.transpose(-1, -2)) * link) @ v
    # what each chunk adds to the state after its last step, padding included, and what of an earlier state it leaves
    add = (k * torch.where(run == run[..., -1:], power(end - at).unsqueeze(1), 0.0).unsqueeze(-1)).transpose(-1, -2) @ v
    last = run[..., -1]                                                               # [N, 1, n]
    order = torch.arange(n, device=q.device)
    over = order.view(-1, 1) - order.view(1, -1)
    into = torch.where((over >= 0) & (last.unsqueeze(-1) == last.unsqueeze(-2)), power(over.clamp(min=0) * chunk), 0.0)     # [N, H, n, n]: from after chunk m to after chunk l
    after = (into @ add.flatten(3)).view(N, H, n, dk, dv)
    after = after + torch.where(last == 0, power(order * chunk + end + entry), 0.0).view(N, H, n, 1, 1) * first.unsqueeze(2)
    before = torch.cat([first.unsqueeze(2), after[:, :, :-1]], 2)
    seen = torch.cat([run.new_zeros(N, 1, 1, 1), run[:, :, :-1, -1:]], 2)             # cuts before the chunk
    reach = power((at + 1).expand(n, chunk) - torch.where(order == 0, 1 - entry, 0).view(-1, 1))
    o = o + torch.where(run == seen, reach, 0.0).unsqueeze(-1) * (q @ before)
    o = o.permute(2, 3, 0, 1, 4).reshape(n * chunk, N, H, dv)[:T]
    # without the padding steps after the last one
    left = ((T - 1) - (n - 1) * chunk)
    add = (k[:, :, -1] * torch.where((run[:, :, -1] == run[:, :, -1, left:left + 1]) & (at <= left), power((left - at).clamp(min=0)).unsqueeze(0), 0.0).unsqueeze(-1)).transpose(-1, -2) @ v[:, :, -1]
    gone = torch.where(run[:, :, -1, left] == seen[:, :, -1, 0], power(torch.tensor(left + (1 if n > 1 else entry), device=q.device)), 0.0)
    return o, add + gone.view(N, H, 1, 1) * before[:, :, -1]


def _plain_attention(s):
    dt = s["q"].dtype
    q, k, v, ld, scale = s["q"].float(), s["k"].float(), s["v"].float(), s["log_decay"], s["scale"]
    T, N = q.shape[:2]
    done = torch.zeros(T, N, device=q.device, dtype=torch.bool) if s["done_in"] is None else s["done_in"] != 0
    cut = torch.cat([torch.zeros_like(done[:1]), done[:-1]])
    keep = (~done[-1]).float().view(N, 1, 1, 1)
    o, last = _memory(q, k, v, ld, cut, s["s0"], 1)
    out = {"o": (scale * o).to(dt), "s_last": last * keep}
    if s["train"]:
        # three memories of the same kind: keys looked up by the gradient, and backwards in time the gradient looked up by
        # the keys and the queries by the values
        do = scale * s["do"].float()
        back, rev = done.flip(0), (do.flip(0), q.flip(0), k.flip(0), v.flip(0))
        out["dq"] = _memory(do, v, k, ld, cut, s["s0"].transpose(-1, -2), 1)[0].to(dt)
        dv, left = _memory(rev[2], rev[1], rev[0], ld, back, s["ds_last"], 0)
        dk, _ = _memory(rev[3], rev[0], rev[1], ld, back, s["ds_last"].transpose(-1, -2), 0)
        out["dk"], out["dv"] = dk.flip(0).to(dt), dv.flip(0).to(dt)
        out["ds0"] = torch.exp(ld).view(1, -1, 1, 1) * left
    return out


def _turn(x, cos, sin, interleaved):
    """The first 2 x pairs entries of x [tokens, heads, dim] turned pair by pair."""
    n = cos.shape[1]
    cos, sin = cos.unsqueeze(1), sin.unsqueeze(1)
    if interleaved:
        a, b = x[..., :2 * n:2], x[..., 1:2 * n:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(2)
    else:
        a, b = x[..., :n], x[..., n:2 * n]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., 2 * n:]], -1)


def _plain_qk(s):
    dt = s["q"].dtype
    angle = s["positions"].double().unsqueeze(1) * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    out = {}
    for n in ("q", "k"):
        x, w = s[n].float(), s["w" + n].float()
        rstd = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
        xhat = x * rstd
        out[n] = _turn(xhat * w, cos, sin, s["interleaved"]).to(dt)
        if s["train"]:
            dy = _turn(s["d" + n].float(), cos, -sin, s["interleaved"])
            wdy = dy * w
            out["d" + n] = (rstd * (wdy - xhat * (wdy * xhat).mean(-1, keepdim=True))).to(dt)
            out["dw" + n] = (dy * xhat).sum((0, 1)).to(s["w" + n].dtype)
    return out


def _plain_adjust(s):
    logits = s["logits"]
    R, V = logits.shape
    x = logits.float()
    if s["history_in"] is not None:
        h = s["history_in"].long()
        live = torch.arange(h.shape[1], device=h.device).unsqueeze(0) < s["lengths"].unsqueeze(1)
        count = torch.zeros(R, V, device=h.device, dtype=torch.int32).scatter_add_(1, h, live.to(torch.int32))
        rep = s["repetition"].unsqueeze(1)
        x = torch.where(count > 0, torch.where(x > 0, x / rep, x * rep), x)
        x = x - s["frequency"].unsqueeze(1) * count - s["presence"].unsqueeze(1) * (count > 0)
    if s["bias_ids"] is not None:
        ids = s["bias_ids"].long()
        x = x + torch.zeros_like(x).scatter_add_(1, ids.clamp(min=0), torch.where(ids >= 0, s["bias_values"], 0.0))
    if s["mask_in"] is not None:
        at = torch.arange(V, device=x.device)
        x = torch.where((s["mask_in"][:, at // 32] >> (at % 32)) & 1 != 0, x, -math.inf)
    return x.to(logits.dtype)


_PLAIN = {"attention": _plain_attention, "qk": _plain_qk, "adjust": _plain_adjust}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    e = 4 if case["dtype"] == "float32" else 2
    if case["op"] == "attention":
        n, dk, dv = case["steps"] * case["batch"] * case["heads"], case["dk"], case["dv"]
        state, flags = 4 * case["batch"] * case["heads"] * dk * dv, case["steps"] * case["batch"] if case["done"] else 0
        moved, ops = n * e * (2 * dk + 2 * dv) + 2 * state + flags, 4 * n * dk * dv
        if case["train"]:     # do, q, k and v read, dq, dk and dv written; s0 and ds_last read, ds0 written
            moved, ops = moved + n * e * (4 * dk + 3 * dv) + 3 * state + flags, ops + 10 * n * dk * dv
        return {"bytes": moved, "flops": ops}
    if case["op"] == "qk":
        n = case["tokens"] * (case["q_heads"] + case["k_heads"]) * case["dim"]
        moved, ops = 2 * n * e + 4 * case["tokens"], 8 * n
        if case["train"]:
            moved, ops = moved + 3 * n * e + 4 * case["tokens"], ops + 16 * n
        return {"bytes": moved, "flops": ops}
    n = case["rows"] * case["vocab"]
    return {"bytes": 2 * n * e + case["rows"] * (2 * case["history"] + 8 * case["biases"]) + (n // 8 if case["mask"] else 0), "flops": 2 * n}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "qk": _exact_qk, "adjust": _exact_adjust}[case["op"]](s)


def _exact_attention(s):
    """Step by step, one matrix a head."""
    q, k, v, scale = s["q"].double(), s["k"].double(), s["v"].double(), s["scale"]
    T, N, H, dk = q.shape
    g = torch.exp(s["log_decay"].double()).view(1, H, 1, 1)
    keep = torch.ones(T, N, 1, 1, 1, device=q.device, dtype=torch.float64)
    if s["done_in"] is not None:
        keep = keep * (s["done_in"] == 0).view(T, N, 1, 1, 1)
    state = s["s0"].double()
    o, dq = torch.empty_like(v), torch.empty_like(q)
    do = s["do"].double() if s["train"] else None
    for t in range(T):
        state = torch.addcmul(g * state, k[t].unsqueeze(-1), v[t].unsqueeze(-2))
        o[t] = scale * torch.matmul(q[t].unsqueeze(-2), state).squeeze(-2)
        if s["train"]:
            dq[t] = scale * torch.matmul(state, do[t].unsqueeze(-1)).squeeze(-1)
        state = state * keep[t]
    out = {"o": o, "s_last": state}
    if s["train"]:
        dk_, dv = torch.empty_like(k), torch.empty_like(v)
        from_later = s["ds_last"].double()
        for t in reversed(range(T)):
            slope = torch.addcmul(from_later * keep[t], q[t].unsqueeze(-1), scale * do[t].unsqueeze(-2))
            dk_[t] = torch.matmul(slope, v[t].unsqueeze(-1)).squeeze(-1)
            dv[t] = torch.matmul(k[t].unsqueeze(-2), slope).squeeze(-2)
            from_later = g * slope
        out["dq"], out["dk"], out["dv"], out["ds0"] = dq, dk_, dv, from_later
    return out


def _exact_qk(s):
    n = s["inv_freq"].shape[0]
    phase = torch.polar(torch.ones(1, 1, 1, dtype=torch.float64, device=s["q"].device),
                        (s["positions"].double().view(-1, 1, 1) * s["inv_freq"].double().view(1, 1, -1)))

    def rotated(x, by):
        pairs = x[..., :2 * n].unflatten(-1, (n, 2)) if s["interleaved"] else x[..., :2 * n].unflatten(-1, (2, n)).transpose(-1, -2)
        z = torch.view_as_real(torch.complex(pairs[..., 0].contiguous(), pairs[..., 1].contiguous()) * by)
        z = z if s["interleaved"] else z.transpose(-1, -2)
        return torch.cat([z.flatten(-2), x[..., 2 * n:]], -1)

    out = {}
    for name in ("q", "k"):
        x, w = s[name].double(), s["w" + name].double()
        d = x.shape[-1]
        ms = x.pow(2).sum(-1, keepdim=True) / d + EPS
        out[name] = rotated(x / ms.sqrt() * w, phase)
        if s["train"]:
            dy = rotated(s["d" + name].double(), phase.conj())
            dms = -0.5 * (dy * w * x).sum(-1, keepdim=True) * ms.pow(-1.5)
            out["d" + name] = dy * w / ms.sqrt() + dms * 2.0 * x / d
            out["dw" + name] = torch.einsum("thd,thd->d", dy, x / ms.sqrt())
    return out


def _exact_adjust(s):
    """Row by row: count, change what was counted, add what is listed, cross out what is not allowed."""
    x = s["logits"].double()
    R, V = x.shape
    for r in range(R):
        if s["history_in"] is not None:
            count = torch.bincount(s["history_in"][r, :int(s["lengths"][r])].long(), minlength=V).double()
            seen = count.nonzero()[:, 0]
            rep, l = float(s["repetition"][r]), x[r, seen]
            x[r, seen] = l * rep ** -torch.sign(l) - float(s["frequency"][r]) * count[seen] - float(s["presence"][r])
        if s["bias_ids"] is not None:
            listed_ = s["bias_ids"][r] >= 0
            x[r].index_add_(0, s["bias_ids"][r][listed_].long(), s["bias_values"][r][listed_].double())
    if s["mask_in"] is not None:
        bits = s["mask_in"].unsqueeze(-1).bitwise_and(torch.bitwise_left_shift(torch.ones(32, device=x.device, dtype=torch.int32), torch.arange(32, device=x.device, dtype=torch.int32)))
        x = x.masked_fill(bits.flatten(1)[:, :V] == 0, -math.inf)
    return x
