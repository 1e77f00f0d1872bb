"""The calls that the language-model operators are measured on.

A case is one pass through one operator: dropout whose mask is a function of a seed, a row's
number and a column (forward with or without a residual, backward); the log-probabilities of given
tokens under rows of logits (forward, backward); the preference loss of pairs of sequences and the
clipped policy loss with a KL term, each from logits to the loss and the logits' gradient.

`run` computes them in elementary torch operations in 32 bits, or, with `own` set, through the
framework's entry points.
"""

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
LOSS_SCALE = {"f32": 1.0, "bf16": 1.0, "f16": 4096.0}   # half precision has few small numbers
BETA, SMOOTHING = 0.1, 0.05              # preference loss
CLIP_LOW, CLIP_HIGH = 0.2, 0.28          # policy loss
MASK64 = (1 << 64) - 1
GAMMA, MIX1, MIX2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB
CHUNK = 1 << 27                          # values that the 64-bit evaluation widens at a time


def listed():
    return [
        # One short sequence through a layer's end (dropout and residual): latency is all.
        dropout("dropout_small", "forward", "bf16", rows=64, cols=1024, residual=True),
        # A partition's samples, gathered in another order than the data set's, with a number of
        # features that divides by nothing.
        dropout("dropout_odd_f32", "forward", "f32", rows=8191, cols=1001, shuffled=True),
        # The backward pass of a wide layer over a large batch of tokens.
        dropout("dropout_backward_large", "backward", "bf16", rows=65536, cols=8192),
        # Rescoring one answer of 32 tokens: a few long rows, latency.
        logprobs("logprobs_small", "forward", "bf16", rows=32, cols=32768),
        # The repository's own classifier: a million samples of 10 classes.
        logprobs("logprobs_classes", "forward", "f32", rows=1048576, cols=10),
        # A fine-tuning step's backward pass: a vocabulary of odd size in padded rows, the prompt's
        # tokens without a loss.
        logprobs("logprobs_backward_odd", "backward", "f16", rows=2047, cols=50021, pad=27, masked=0.25),
        # The reference model's scores of a large batch.
        logprobs("logprobs_large", "forward", "bf16", rows=16384, cols=131072),
        # Four pairs of short answers and a small vocabulary.
        preference("preference_small", "f32", rows=96, cols=1000, pairs=4),
        # A batch of 16 pairs of unequal lengths, a third of the tokens belonging to prompts.
        preference("preference_pairs", "bf16", rows=12289, cols=50021, pairs=16, masked=0.33, banned=True),
        # One short sampled answer.
        policy("policy_small", "f32", rows=64, cols=32768),
        # An ordinary batch of sampled answers.
        policy("policy_batch", "f16", rows=4096, cols=65536, masked=0.1, banned=True),
        # A large one, on a vocabulary whose rows start at no alignment.
        policy("policy_large_odd", "bf16", rows=8192, cols=131071),
    ]


def dropout(name, direction, dtype, rows, cols, p=0.1, residual=False, shuffled=False):
    return dict(name=name, op="dropout", direction=direction, dtype=dtype, rows=rows, cols=cols, p=p,
                residual=residual, shuffled=shuffled)


def logprobs(name, direction, dtype, rows, cols, pad=0, masked=0.0, banned=False):
    return dict(name=name, op="logprobs", direction=direction, dtype=dtype, rows=rows, cols=cols, pad=pad,
                masked=masked, banned=banned)


def preference(name, dtype, rows, cols, pairs, pad=0, masked=0.0, banned=False):
    return dict(name=name, op="preference", dtype=dtype, rows=rows, cols=cols, pairs=pairs, pad=pad,
                masked=masked, banned=banned)


def policy(name, dtype, rows, cols, pad=0, masked=0.0, banned=False, kl=0.04):
    return dict(name=name, op="policy", dtype=dtype, rows=rows, cols=cols, pad=pad, masked=masked,
                banned=banned, kl=kl)


def draw(rng):
    """A case of the listed ones' ranges: values, columns and rows over their logarithms."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["dropout", "logprobs", "preference", "policy"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    most = (1 << 29) // (2 if dtype == "f32" else 1)
    values = log_int(1 << 12, most)
    if op == "dropout":
        cols = log_int(64, 8192)
        rows = max(1, min(values // cols, 1 << 20))
        direction = rng.choice(["forward", "backward"])
        case = dropout("", direction, dtype, rows, cols, p=rng.choice([0.05, 0.1, 0.2, 0.5]),
                       residual=direction == "forward" and rng.random() < 0.5, shuffled=rng.random() < 0.5)
    else:
        cols = log_int(10, 131072)
        rows = max(1, min(values // cols, 1 << 20))
        pad = rng.choice([0, 0, rng.randint(1, 64)])
        masked = rng.choice([0.0, 0.1, 0.33])
        banned = cols >= 1000 and rng.random() < 0.5
        if op == "logprobs":
            case = logprobs("", rng.choice(["forward", "backward"]), dtype, rows, cols, pad, masked, banned)
        elif op == "policy":
            case = policy("", dtype, rows, cols, pad, masked, banned, kl=rng.choice([0.0, 0.04]))
        else:
            case = preference("", dtype, rows, cols, rng.randint(1, max(1, min(rows // 8, 64))), pad, masked, banned)
    del case["name"]
    return case


def logits_of(case, gen, device):
    """Rows of logits as a trained model gives them: a spread of a few units with the token that
    follows ahead, reserved tokens at -inf, and rows that may be padded."""
    rows, cols, dtype = case["rows"], case["cols"], DTYPES[case["dtype"]]
    z = torch.randn(rows, cols + case["pad"], generator=gen, device=device, dtype=dtype)[:, :cols]
    z.mul_(2.0)
    y = torch.randint(0, cols, (rows,), generator=gen, device=device)
    at = torch.arange(rows, device=device)
    ahead = (z[at, y].float() + math.log(cols)).to(dtype)
    if case["banned"]:
        reserved = torch.rand(cols, generator=gen, device=device) < 0.01
        z.masked_fill_(reserved, -math.inf)
    z[at, y] = ahead
    return z, y.to(torch.int32)


def token_logprobs_of(z, y):
    """Log-probabilities of the tokens y, a block of rows at a time."""
    out = torch.empty(z.shape[0], device=z.device)
    step = max(1, CHUNK // z.shape[1])
    for a in range(0, z.shape[0], step):
        x = z[a:a + step].float()
        out[a:a + step] = x.gather(1, y[a:a + step].long()[:, None])[:, 0] - torch.logsumexp(x, 1)
    return out


def prepare(case, seed):
    device = torch.device("cuda")
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    rows, cols = case["rows"], case["cols"]
    s = dict(case)
    if case["op"] == "dropout":
        dtype = DTYPES[case["dtype"]]
        s["x"] = torch.randn(rows, cols, generator=gen, device=device, dtype=dtype)
        s["residual_in"] = (torch.randn(rows, cols, generator=gen, device=device, dtype=dtype)
                            if case["residual"] else None)
        # The numbers of the rows in the data set: consecutive, or gathered from all over it.
        s["first_row"] = int(torch.randint(0, 1 << 40, (1,), generator=gen, device=device))
        s["row_ids"] = (torch.randint(0, 1 << 40, (rows,), generator=gen, device=device)
                        if case["shuffled"] else None)
        s["seed"] = (int(torch.randint(0, 1 << 62, (1,), generator=gen, device=device)) * 4 + 3) & MASK64
        return s
    z, y = logits_of(case, gen, device)
    s["logits"], n_masked, loss_scale = z, int(case["masked"] * rows), LOSS_SCALE[case["dtype"]]
    noise = torch.rand(rows, generator=gen, device=device) * 2 - 1
    if case["op"] == "preference":
        # 2 * pairs sequences of unequal lengths; the first tokens of each are its prompt's.
        seqs = 2 * case["pairs"]
        share = torch.rand(seqs, generator=gen, device=device).add_(0.25).double()
        ends = (share.cumsum(0) / share.sum() * rows).round().to(torch.int64).clamp_(max=rows)
        ends[-1] = rows
        s["offsets"] = torch.cat([ends.new_zeros(1), ends]).to(torch.int32)
        at = torch.arange(rows, device=device)
        seq = torch.searchsorted(ends, at, right=True)
        start = s["offsets"].long()[seq]
        length = s["offsets"].long()[seq + 1] - start
        s["ref"] = token_logprobs_of(z, y) + 0.2 * noise
        y[(at - start) < (case["masked"] * length).floor()] = -1
        s["targets"], s["scale"] = y, loss_scale / case["pairs"]
        return s
    lp = token_logprobs_of(z, y)
    y[torch.randperm(rows, generator=gen, device=device)[:n_masked]] = -1
    s["targets"] = y
    if case["op"] == "logprobs":
        if case["direction"] == "backward":
            x = z.float()
            top = x.amax(1)
            log_sum = torch.logsumexp(x, 1).double() - top.double()
            s["stats"] = torch.stack([top, log_sum.float()], 1)
            s["grad"] = noise * (loss_scale / rows)
        return s
    # The sampling policy's log-probabilities lie a little off the present ones. No ratio stands
    # within 0.002 of a clip bound, where the gradient jumps and rounding would decide.
    shift = 0.6 * noise
    for bound in (math.log(1 - CLIP_LOW), math.log(1 + CLIP_HIGH)):
        shift = torch.where((shift - bound).abs() < 0.002, shift + 0.004, shift)
    s["old"] = lp - shift
    s["ref"] = lp + 0.3 * (torch.rand(rows, generator=gen, device=device) * 2 - 1)
    s["advantages"] = torch.randn(rows, generator=gen, device=device)
    s["scale"] = loss_scale / rows
    return s


def run(state):
    return (run_own if own else run_plain)(state)


def run_own(s):
    from paper_2607_20739_amd import ops
    if s["op"] == "dropout":
        if s["direction"] == "forward":
            return ops.dropout(s["x"], s["p"], s["seed"], residual=s["residual_in"], row_ids=s["row_ids"],
                               first_row=s["first_row"])
        return ops.dropout_backward(s["x"], s["p"], s["seed"], row_ids=s["row_ids"], first_row=s["first_row"])
    if s["op"] == "logprobs":
        if s["direction"] == "forward":
            return ops.token_logprobs(s["logits"], s["targets"])
        return ops.token_logprobs_backward(s["logits"], s["targets"], s["stats"], s["grad"])
    if s["op"] == "preference":
        return ops.preference_loss(s["logits"], s["targets"], s["offsets"], s["ref"], beta=BETA,
                                   label_smoothing=SMOOTHING, scale=s["scale"])
    return ops.policy_loss(s["logits"], s["targets"], s["old"], s["advantages"], ref_logprobs=s["ref"],
                           clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl=s["kl"], scale=s["scale"])


# ---- the plain forms ------------------------------------------------------------------------

def signed(v):
    """The 64-bit pattern v as torch's int64 holds it."""
    v &= MASK64
    return v - (1 << 64) if v >> 63 else v


def mix64(z):
    """SplitMix64's finaliser on int64 tensors (products wrap; shifts are made logical)."""
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * signed(MIX1)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * signed(MIX2)
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def kept(s):
    """The mask: value j of row r is kept where the 16 bits that belong to it reach the threshold."""
    rows, cols, device = s["rows"], s["cols"], s["x"].device
    ids = s["row_ids"]
    if ids is None:
        ids = s["first_row"] + torch.arange(rows, device=device)
    key = mix64(signed(s["seed"]) + (ids + 1) * signed(GAMMA))
    word = torch.arange((cols + 3) // 4, device=device)
    bits = mix64(key[:, None] + (word + 1) * signed(GAMMA))
    fields = torch.stack([(bits >> (16 * k)) & 0xFFFF for k in range(4)], 2).reshape(rows, -1)[:, :cols]
    return fields >= threshold(s["p"])


def threshold(p):
    return int(math.floor(p * 65536 + 0.5))


def run_plain(s):
    if s["op"] == "dropout":
        factor = 65536.0 / (65536 - threshold(s["p"]))
        y = torch.where(kept(s), s["x"].float() * factor, 0.0)
        if s["residual_in"] is not None:
            y = y + s["residual_in"].float()
        return y.to(s["x"].dtype)
    z, counts = s["logits"].float(), s["targets"] >= 0
    y = s["targets"].clamp(min=0).long()[:, None]
    if s["op"] == "logprobs" and s["direction"] == "backward":
        p = torch.exp(z - s["stats"][:, :1] - s["stats"][:, 1:])
        g = torch.where(counts, s["grad"], 0.0)
        return logits_gradient(p, y, g).to(s["logits"].dtype)
    top = z.amax(1)
    e = torch.exp(z - top[:, None])
    total = e.sum(1)
    lp = torch.where(counts, (z.gather(1, y)[:, 0] - top) - torch.log(total), 0.0)
    if s["op"] == "logprobs":
        stats = torch.stack([top, torch.log(total)], 1)
        return lp, torch.where(counts[:, None], stats, 0.0)
    p = e / total[:, None]
    if s["op"] == "preference":
        # Sequence sums by differences of a running sum; the running sum itself in 64 bits.
        each = torch.where(counts, lp - s["ref"], 0.0).double()
        running = torch.cat([each.new_zeros(1), each.cumsum(0)])
        o = s["offsets"].long()
        sums = (running[o[1:]] - running[o[:-1]]).float()
        h = BETA * (sums[0::2] - sums[1::2])
        loss = (1 - SMOOTHING) * softplus(-h) + SMOOTHING * softplus(h)
        slope = (torch.sigmoid(h) - (1 - SMOOTHING)) * (BETA * s["scale"])
        per_seq = torch.stack([slope, -slope], 1).reshape(-1)
        g = per_seq.repeat_interleave(o[1:] - o[:-1], output_size=s["rows"])
        return loss, h, lp, logits_gradient(p, y, torch.where(counts, g, 0.0)).to(s["logits"].dtype)
    ratio = torch.exp(lp - s["old"])
    a = s["advantages"]
    free, bound = ratio * a, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a
    d = s["ref"] - lp
    loss = torch.maximum(-free, -bound) + s["kl"] * (torch.expm1(d) - d)
    slope = torch.where(free <= bound, -free, 0.0) - s["kl"] * torch.expm1(d)
    g = torch.where(counts, slope * s["scale"], 0.0)
    return torch.where(counts, loss, 0.0), lp, logits_gradient(p, y, g).to(s["logits"].dtype)


def softplus(x):
    return x.clamp(min=0) + torch.log1p(torch.exp(-x.abs()))


def logits_gradient(p, y, g):
    """g (onehot(y) - p), row by row."""
    dz = p * -g[:, None]
    return dz.scatter_add_(1, y, g[:, None])


# ---- the definitions in 64 bits -------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return exact_dropout(s) if s["op"] == "dropout" else exact_logits(s)


def times64(lo, hi, c):
    """(lo, hi) * c mod 2^64, in halves of 32 bits built from products of 16 by 32 bits."""
    c_lo, c_hi, m32 = c & 0xFFFFFFFF, c >> 32, 0xFFFFFFFF
    low = (lo & 0xFFFF) * c_lo
    mid = (lo >> 16) * c_lo
    low_sum = low + ((mid & 0xFFFF) << 16)
    carry = (low_sum >> 32) + (mid >> 16)

    def low32(a, b):        # a * b mod 2^32
        return ((a & 0xFFFF) * b + ((((a >> 16) * b) & 0xFFFF) << 16)) & m32
    return low_sum & m32, (carry + low32(hi, c_lo) + low32(lo, c_hi)) & m32


def finalise(lo, hi):
    """SplitMix64's finaliser on halves of 32 bits."""
    for shift, c in ((30, MIX1), (27, MIX2), (31, None)):
        s_lo = ((lo >> shift) | (hi << (32 - shift))) & 0xFFFFFFFF
        lo, hi = lo ^ s_lo, hi ^ (hi >> shift)
        if c is not None:
            lo, hi = times64(lo, hi, c)
    return lo, hi


def draw_words(base_lo, base_hi, index):
    """Outputs `index` (below 2^41) of the streams seeded with (base_lo, base_hi)."""
    n = index + 1
    g_lo, g_hi = times64(n & 0xFFFFFFFF, n >> 32, GAMMA)
    lo = base_lo + g_lo
    return finalise(lo & 0xFFFFFFFF, (base_hi + g_hi + (lo >> 32)) & 0xFFFFFFFF)


def exact_dropout(s):
    rows, cols, device = s["rows"], s["cols"], s["x"].device
    out = torch.empty(rows, cols, dtype=torch.float64, device=device)
    keep_share = 1.0 - threshold(s["p"]) / 65536.0
    column = torch.arange(cols, device=device)
    step = max(1, CHUNK // cols)
    for a in range(0, rows, step):
        b = min(rows, a + step)
        ids = (torch.arange(s["first_row"] + a, s["first_row"] + b, device=device) if s["row_ids"] is None
               else s["row_ids"][a:b])
        k_lo, k_hi = draw_words(torch.full_like(ids, s["seed"] & 0xFFFFFFFF), torch.full_like(ids, s["seed"] >> 32), ids)
        words = torch.arange((cols + 3) // 4, device=device)[None, :]
        lo, hi = draw_words(k_lo[:, None], k_hi[:, None], words)
        half = torch.where((column % 4 < 2)[None, :], lo[:, column // 4], hi[:, column // 4])
        u = torch.where((column % 2 == 0)[None, :], half % 65536, half // 65536).double() / 65536.0
        v = s["x"][a:b].double() / keep_share
        v = v * (u >= threshold(s["p"]) / 65536.0)
        out[a:b] = v if s["residual_in"] is None else v + s["residual_in"][a:b].double()
    return out


def exact_logits(s):
    rows, cols, device = s["rows"], s["cols"], s["logits"].device
    y, on = s["targets"].long(), s["targets"] >= 0
    step = max(1, CHUNK // cols)
    blocks = [(a, min(rows, a + step)) for a in range(0, rows, step)]
    top, log_sum, at_target = (torch.zeros(rows, dtype=torch.float64, device=device) for _ in range(3))
    for a, b in blocks:
        x = s["logits"][a:b].double()
        top[a:b] = x.max(1).values
        log_sum[a:b] = torch.log(torch.exp(x - top[a:b, None]).sum(1))
        at_target[a:b] = x[torch.arange(b - a, device=device), y[a:b].clamp(min=0)]
    lp = (at_target - top - log_sum) * on

    def gradient(g):
        out = torch.empty(rows, cols, dtype=torch.float64, device=device)
        t = torch.arange(rows, device=device)
        for a, b in blocks:
            x = s["logits"][a:b].double()
            out[a:b] = -torch.exp(x - (top + log_sum)[a:b, None]) * (g * on)[a:b, None]
        out[t[on], y[on]] += g[on]
        return out

    if s["op"] == "logprobs":
        if s["direction"] == "forward":
            return lp, torch.stack([top * on, log_sum * on], 1)
        top, log_sum = s["stats"][:, 0].double(), s["stats"][:, 1].double()
        return gradient(s["grad"].double())
    if s["op"] == "preference":
        margin, loss, g = [], [], torch.zeros(rows, dtype=torch.float64, device=device)
        o = s["offsets"].tolist()
        score = (lp - s["ref"].double()) * on
        for i in range(s["pairs"]):
            won, lost = slice(o[2 * i], o[2 * i + 1]), slice(o[2 * i + 1], o[2 * i + 2])
            h = BETA * float(score[won].sum() - score[lost].sum())
            sure = 1.0 / (1.0 + math.exp(-h)) if h > -700 else 0.0
            not_sure = 1.0 / (1.0 + math.exp(h)) if h < 700 else 0.0
            margin.append(h)
            loss.append((1 - SMOOTHING) * (max(-h, 0) + math.log1p(math.exp(-abs(h)))) +
                        SMOOTHING * (max(h, 0) + math.log1p(math.exp(-abs(h)))))
            slope = BETA * s["scale"] * (SMOOTHING * sure - (1 - SMOOTHING) * not_sure)
            g[won], g[lost] = slope, -slope
        return (torch.tensor(loss, dtype=torch.float64), torch.tensor(margin, dtype=torch.float64), lp, gradient(g))
    ratio, a = torch.exp(lp - s["old"].double()), s["advantages"].double()
    # Clipped: above the upper bound with a positive advantage, below the lower with a negative one.
    clipped = ((a > 0) & (ratio > 1 + CLIP_HIGH)) | ((a < 0) & (ratio < 1 - CLIP_LOW))
    limit = torch.where(a > 0, 1.0 + CLIP_HIGH, 1.0 - CLIP_LOW)
    off = torch.exp(s["ref"].double() - lp)
    loss = -torch.where(clipped, limit, ratio) * a + s["kl"] * (off - torch.log(off) - 1)
    slope = torch.where(clipped, 0.0, -ratio * a) + s["kl"] * (1 - off)
    return loss * on, lp, gradient(slope * s["scale"])


def work(case):
    """Bytes that have to move, and operations: rows without a token are written, not read."""
    b, rows, cols = BYTES[case["dtype"]], case["rows"], case["cols"]
    values = rows * cols
    if case["op"] == "dropout":
        ids = 8 * rows if case["shuffled"] else 0
        # Two 64-bit products and nine further operations for 4 values, then compare, select, scale.
        return {"bytes": b * values * (3 if case["residual"] else 2) + ids, "flops": values * 6}
    read = b * cols * (rows - int(case["masked"] * rows))
    if case["op"] == "logprobs" and case["direction"] == "forward":
        return {"bytes": read + (4 + 12) * rows, "flops": 4 * values}
    if case["op"] == "logprobs":
        return {"bytes": read + b * values + (4 + 12) * rows, "flops": 4 * values}
    if case["op"] == "preference":
        return {"bytes": read + b * values + 12 * rows, "flops": 8 * values}
    return {"bytes": read + b * values + 24 * rows, "flops": 8 * values}
