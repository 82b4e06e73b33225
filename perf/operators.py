"""Training against a target's top logits: what is measured of it, and the same in plain torch.

Three operators that work together: a target row's k largest logits with the log-sum-exp of the
rest (aal_topk_logits), the acceptance-aware objectives against such lists with their gradient
(aal_topk_loss_fwd_bwd), and the penalties, biases and grammar masks that draft and target logits
go through before they are compared, with the gradient through them (aal_logits_process and
aal_logits_process_bwd).

listed() names representative calls, draw() gives more of the same ranges, prepare() makes what a
program has in hand, run() is one pass, work() what no implementation can avoid, exact() the same
results in 64 bits.

Ranges: vocabularies of 1,000 to 152,000 entries (two thirds of them padded to a multiple of 16),
lists of 1 to 256 logits, windows of 1 to 16 positions, histories of 0 to 32,768 tokens, from a few
thousand logits per call up to the 1.84e9 of 2048 windows x 7 positions x 128,256.
"""
import math

import torch

from paper_2609_24150_amd.inputs import make_logits

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp32": 4}
MOST_ELEMENTS = 2048 * 7 * 128256

# (wtv, eal, kl, tv) weights of the training objectives
WEIGHTS = {
    "wtv": (1.0, 0.0, 0.0, 0.0),
    "eal": (0.0, 1.0, 0.0, 0.0),
    "kl": (0.0, 0.0, 1.0, 0.0),
    "kl+eal": (0.0, 0.1, 1.0, 0.0),
    "kl+tv": (0.0, 0.0, 1.0, 1.0),
}


def listed():
    return [
        # The smallest extraction, bound by latency: a unit-test sized batch in fp32.
        dict(name="topk-small", op="topk", rows=256, V=1024, k=8, dtype="fp32", recipe="c1", T=1.0),
        # One draft window while serving: few rows of the largest vocabulary.
        dict(name="topk-window", op="topk", rows=7, V=151936, k=20, dtype="bf16", recipe="c3", T=1.0),
        # Storing the target's lists for a full training batch.
        dict(name="topk-teacher", op="topk", rows=14336, V=128256, k=64, dtype="bf16", recipe="c2", T=1.0),
        # Short sequences over an unpadded vocabulary, longer lists, low temperature.
        dict(name="topk-ragged", op="topk", rows=768, V=50001, k=100, dtype="bf16", recipe="c3", T=0.7),
        # The smallest loss call, bound by latency and launches.
        dict(name="loss-small", op="loss", B=64, S=4, K=4, V=1024, k=8, dtype="fp32", recipe="c1", weights="kl+eal",
             td=1.0, tt=1.0, sequences=False, rest=True),
        # The training step at full batch: window total variation over disjoint windows.
        dict(name="loss-wtv-train", op="loss", B=2048, S=7, K=7, V=128256, k=64, dtype="bf16", recipe="c2",
             weights="wtv", td=1.0, tt=1.0, sequences=False, rest=True),
        # The anchored greedy recipe over sequences with windows sliding by one.
        dict(name="loss-kl-eal-sliding", op="loss", B=2, S=1024, K=7, V=128256, k=128, dtype="bf16", recipe="c2",
             weights="kl+eal", td=1.0, tt=1.0, sequences=True, rest=True),
        # The anchored sampling recipe over lists cut to a nucleus, without a remainder, unpadded vocabulary.
        dict(name="loss-kl-tv-ragged", op="loss", B=8, S=96, K=5, V=50001, k=100, dtype="bf16", recipe="c3",
             weights="kl+tv", td=0.7, tt=0.7, sequences=True, rest=False, cut=True),
        # One decoding step of four requests: penalties over their histories and a grammar.
        dict(name="process-decode", op="process", N=4, K=1, V=128256, dtype="bf16", recipe="c2", hist=4096,
             masks=4, bias=16),
        # A training batch: the rows of a window share the context that their histories extend.
        dict(name="process-train", op="process", N=512, K=7, V=128256, dtype="bf16", recipe="c2", hist=1024, masks=64,
             bias=0),
        # The gradient through the processing of that batch.
        dict(name="process-bwd-train", op="process_bwd", N=512, K=7, V=128256, dtype="bf16", recipe="c2", hist=1024,
             masks=64, bias=0),
        # The same over an unpadded vocabulary in fp32, with biases and long histories.
        dict(name="process-bwd-ragged", op="process_bwd", N=96, K=8, V=50001, dtype="fp32", recipe="c3", hist=8192,
             masks=8, bias=100),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["topk", "topk", "loss", "loss", "loss", "process", "process", "process_bwd"])
    V = _log(rng, 1000, 152000)
    if rng.random() < 2 / 3:
        V = V // 16 * 16
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    recipe = rng.choice(["c1", "c2", "c3", "c4"])
    most = MOST_ELEMENTS // (2 if dtype == "fp32" else 1)
    c = dict(op=op, V=V, dtype=dtype, recipe=recipe)
    if op == "topk":
        c.update(rows=max(1, _log(rng, 1 << 12, most) // V), k=_log(rng, 1, 256), T=rng.choice([1.0, 1.0, 0.7, 0.5]))
    elif op == "loss":
        K = rng.choice([1, 2, 3, 4, 5, 6, 7, 7, 8, 8, 9, 12, 16])
        rows = max(K, _log(rng, 1 << 12, most) // V)
        seq = rng.random() < 0.7
        S = rng.randint(K, max(K, min(2048, rows))) if seq else K
        T = rng.choice([1.0, 1.0, 0.7, 0.5])
        c.update(B=max(1, rows // S), S=S, K=K, k=_log(rng, 1, 256), weights=rng.choice(sorted(WEIGHTS)), td=T, tt=T,
                 sequences=seq, rest=rng.random() < 0.75, cut=rng.random() < 0.3, grad=rng.random() < 0.85)
        if dtype == "bf16" and rng.random() < 0.2:
            c["grad_dtype"] = "fp32"
    else:
        K = rng.choice([1, 1, 4, 7, 8])
        rows = max(K, _log(rng, 1 << 12, most // 4) // V)
        N = max(1, rows // K)
        # at most 2^25 history entries over all rows
        hist = rng.choice([0, 1, 1, 1]) * _log(rng, 1, max(1, min(32768, (1 << 25) // (N * K))))
        c.update(N=N, K=K, hist=hist, masks=rng.choice([0, 1, 8, 64]), bias=rng.choice([0, 0, 16, 100]))
    return c


# ----------------------------------------------------------------- inputs
def _generator(seed, stream, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed * 15485863 + stream)
    return g


def _rows(c):
    return c["rows"] if c["op"] == "topk" else c["B"] * c["S"] if c["op"] == "loss" else c["N"] * c["K"]


def _logits(c, seed):
    """(z_draft, z_target) rows of the case's recipe."""
    return make_logits(c["recipe"], (_rows(c), c["V"]), DTYPES[c["dtype"]], seed=seed, chunk_elems=1 << 28)


def _lists(c, zt, seed):
    """The stored lists of target rows: logits, ids and the remainder, as a data set holds them."""
    R, V, k = zt.shape[0], c["V"], c["k"]
    out = _plain_topk(zt, k, c["tt"])
    top, ids = out["logits"], out["ids"]
    if c.get("cut"):
        # cut to a nucleus of another length in each row; a twentieth of the rows (a prompt's) have none
        g = _generator(seed, 3)
        n = (torch.rand(R, generator=g, device=zt.device) * k).long() + 1
        n[torch.rand(R, generator=g, device=zt.device) < 0.05] = 0
        gone = torch.arange(k, device=zt.device)[None, :] >= n[:, None]
        top = top.masked_fill(gone, -math.inf)
        ids = ids.masked_fill(gone, -1)
    return top, ids, out["rest"] if c["rest"] else None


def _rules(c, seed, device="cuda"):
    """Histories, penalties, biases and grammars of the rows of N contexts x K positions."""
    N, K, V, hist = c["N"], c["K"], c["V"], c["hist"]
    R = N * K
    g = _generator(seed, 5, device)
    rand = lambda *s: torch.rand(*s, generator=g, device=device)  # noqa: E731
    pick = lambda values, n: torch.tensor(values, device=device)[(rand(n) * len(values)).long()]  # noqa: E731
    r = {}
    if hist:
        # a context's tokens and the drafted ones after it, frequent words more often
        width = hist + K - 1
        word = torch.exp(rand(N * width) * math.log(V)).long() - 1
        r["tokens"] = (word.clamp_(0, V - 1) * 7919 % V).int()
        context = hist - (rand(N) * rand(N) * hist).long()
        start = torch.arange(N, device=device) * width
        r["hist_start"] = start.repeat_interleave(K)
        r["hist_len"] = (context[:, None] + torch.arange(K, device=device)).reshape(-1).int()
        r["prompt_len"] = (context // 2).repeat_interleave(K).int()
        r["repetition"] = pick([1.0, 1.1, 1.2, 1.3], N).repeat_interleave(K).contiguous()
        r["frequency"] = pick([0.0, 0.2, 0.5], N).repeat_interleave(K).contiguous()
        r["presence"] = pick([0.0, 0.3], N).repeat_interleave(K).contiguous()
    if c["bias"]:
        n = (rand(R) * (c["bias"] + 1)).long()
        r["bias_offsets"] = torch.cat([n.new_zeros(1), n.cumsum(0)])
        at = torch.arange(c["bias"], device=device)
        ids = (at[None, :] * (V // c["bias"]) + (rand(R, 1) * (V // c["bias"])).long()).int()
        keep = at[None, :] < n[:, None]
        r["bias_ids"] = ids[keep]
        r["bias_values"] = ((rand(R, c["bias"]) - 0.5) * 20)[keep]
    if c["masks"]:
        # grammars that leave a few tokens, some or most of them; one of many is at its end and leaves none
        words, M = (V + 31) // 32, c["masks"]
        share = pick([0.0005, 0.05, 0.5, 0.95], M)
        bits = rand(M, words * 32) < share[:, None]
        bits[:, 7 % V] = True
        if M > 32:
            bits[M // 2] = False
        two = torch.ones(32, dtype=torch.int64, device=device) << torch.arange(32, device=device)
        r["mask"] = (bits.view(M, words, 32) * two).sum(-1).int()
        r["mask_row"] = ((rand(R) * 2 * M).long() - M).clamp_(min=-1).int()
    return r


def prepare(case, seed):
    c = case
    zd, zt = _logits(c, seed)
    if c["op"] == "topk":
        return {"case": c, "z": zt}
    if c["op"] == "loss":
        top, ids, rest = _lists(c, zt, seed)
        lead = (c["B"], c["S"])
        return {"case": c, "z": zd.view(*lead, -1), "top": top.view(*lead, -1), "ids": ids.view(*lead, -1),
                "rest": None if rest is None else rest.view(lead)}
    st = {"case": c, "z": zd, "rules": _rules(c, seed)}
    if c["op"] == "process_bwd":
        st["grad"] = torch.randn(zd.shape, generator=_generator(seed, 9), device=zd.device).to(zd.dtype)
    return st


def run(state):
    c = state["case"]
    if c["op"] == "topk":
        return _own_topk(state) if own else _plain_topk(state["z"], c["k"], c["T"])
    if c["op"] == "loss":
        return _own_loss(state) if own else _plain_loss(c, state["z"], state["top"], state["ids"], state["rest"])
    if c["op"] == "process":
        return _own_process(state) if own else _plain_process(c, state["z"], state["rules"])
    return _own_process_bwd(state) if own else _plain_process_bwd(c, state["z"], state["grad"], state["rules"])


# ------------------------------------------------- the framework's operators
def _own_topk(state):
    import paper_2609_24150_amd as aal
    c = state["case"]
    return aal.aal_topk_logits(state["z"], c["k"], c["T"])


def _own_loss(state):
    import paper_2609_24150_amd as aal
    c = state["case"]
    layout = aal.AAL_LAYOUT_SEQUENCES if c["sequences"] else aal.AAL_LAYOUT_WINDOWS
    return aal.aal_topk_loss_fwd_bwd(state["z"], state["top"], state["ids"], c["K"], rest=state["rest"],
                                     weights=WEIGHTS[c["weights"]], temp_draft=c["td"], temp_target=c["tt"],
                                     layout=layout, grad=c.get("grad", True),
                                     grad_dtype=DTYPES[c.get("grad_dtype", c["dtype"])])


def _own_process(state):
    import paper_2609_24150_amd as aal
    return aal.aal_logits_process(state["z"], **state["rules"])


def _own_process_bwd(state):
    import paper_2609_24150_amd as aal
    return aal.aal_logits_process_bwd(state["grad"], state["z"], **state["rules"])


# ---------------------------------------------------------------- plain torch
def _lse(x):
    """ln sum exp of the last dimension, -inf where nothing is finite."""
    m = x.amax(-1)
    s = (x - torch.where(m == -math.inf, 0.0, m)[..., None]).exp_().sum(-1)
    return torch.where(m == -math.inf, 0.0, m) + s.log()


def _plain_topk(z, k, T):
    V = z.shape[-1]
    # one whole number for each entry that orders by value, then by the lower index
    b = (z.float() + 0.0).view(torch.int32)
    b = b ^ ((b >> 31) & 0x7FFFFFFF)
    key = (b.long() << 32) | (V - 1 - torch.arange(V, device=z.device))
    ids = V - 1 - (key.topk(k, -1).values & 0xFFFFFFFF)
    rest = _lse(z.float().scatter(-1, ids, -math.inf).div_(T))
    return {"logits": z.gather(-1, ids), "ids": ids.int(), "rest": rest}


def _windows(a, c):
    """E of every window and dE/da summed over the windows that contain each row, for a [B, S]."""
    K = c["K"]
    w = a.unfold(1, K, 1)  # [B, W, K]: one window where S = K
    if w.shape[1] == 0:
        return a.new_zeros(0), torch.zeros_like(a)
    pre = torch.cat([torch.ones_like(w[..., :1]), w[..., :-1]], -1).cumprod(-1)
    # prod_{l=j+1..i} a_l for j <= i: cumulative products of rows that hold a_l right of the diagonal
    j = torch.arange(K, device=a.device)
    part = torch.where(j[None, :] > j[:, None], w[..., None, :], 1.0).cumprod(-1)
    d = pre * (part * (j[None, :] >= j[:, None])).sum(-1)
    at = torch.arange(w.shape[1], device=a.device)[:, None] + j
    rows = torch.zeros_like(a).index_add_(1, at.reshape(-1), d.flatten(1))
    return (pre * w).sum(-1).flatten(), rows


def _plain_loss(c, z, top, ids, rest):
    B, S, V = z.shape
    w_wtv, w_eal, w_kl, w_tv = WEIGHTS[c["weights"]]
    valid = (ids >= 0) & (ids < V) & (top > -math.inf)
    at = torch.where(valid, ids, 0).long()
    # the target: the list and the remainder as one more entry
    t = torch.where(valid, top.float() / c["tt"], -math.inf)
    t = torch.cat([t, torch.full_like(t[..., :1], -math.inf) if rest is None else rest.float()[..., None]], -1)
    lt = _lse(t)
    empty = lt == -math.inf
    p = torch.where(empty[..., None], 0.0, (t - torch.where(empty, 0.0, lt)[..., None]).exp())
    # the draft: the same entries of its softmax, the remainder summed over the others
    x = z.float() / c["td"]
    x -= x.amax(-1, keepdim=True)
    xi = torch.where(valid, x.gather(-1, at), -math.inf)
    e = x.exp_()
    s = e.sum(-1, keepdim=True)
    # an entry that is no part of the list names a place past the row, which is cut off again
    past = torch.where(valid, ids, V).long()
    listed_ = torch.zeros(B, S, V + 1, dtype=torch.bool, device=z.device).scatter_(-1, past, True)[..., :V]
    er = torch.where(listed_, 0.0, e).sum(-1, keepdim=True)
    q = torch.cat([torch.where(valid, e.gather(-1, at), 0.0), er if rest is not None else torch.zeros_like(er)], -1) / s
    lq = torch.cat([xi, er.log()], -1) - s.log()
    below = (q < p).float()
    a_tv = torch.minimum(p, q).sum(-1)
    qlt = (q * below).sum(-1)
    kl = torch.where(p > 0, p * ((t - lt[..., None]) - lq), 0.0).sum(-1)
    # the greedy token: the largest listed logit, the lower id on ties
    best = torch.where(valid, top.float(), -math.inf).amax(-1, keepdim=True)
    star = torch.where(valid & (top.float() == best), ids, V).amin(-1)
    has = star < V
    is_star = valid & (ids == star[..., None])
    a_eal = (q[..., :-1] * is_star).sum(-1)
    E_tv, d_tv = _windows(a_tv, c)
    E_eal, d_eal = _windows(a_eal, c)
    W = max(1, S - c["K"] + 1) * B
    count = _count(c, B, S, z.device)
    terms = torch.stack([-E_tv.sum() / W, -E_eal.sum() / W, kl.sum() / (B * S),
                         (count * (1 - a_tv)).sum() / (W * c["K"])])
    used = torch.tensor([float(w != 0) for w in WEIGHTS[c["weights"]]], device=z.device)
    terms = torch.where(used > 0, terms, 0.0)
    loss = (terms * torch.tensor(WEIGHTS[c["weights"]], device=z.device)).sum().reshape(1)
    grad = None
    if c.get("grad", True):
        g_tv = (-w_wtv * d_tv - w_tv * count / c["K"]) / W / c["td"]
        g_eal = -w_eal * d_eal / W / c["td"] * a_eal
        g_kl = torch.where(empty, 0.0, w_kl / (B * S) / c["td"])
        ratio = torch.where(q[..., -1] > 0, p[..., -1] / q[..., -1], 0.0)
        others = g_tv * (below[..., -1] - qlt) - g_eal + g_kl * (1 - ratio)
        mine = (q * (g_tv[..., None] * (below - qlt[..., None]) - g_eal[..., None] + g_kl[..., None])
                - g_kl[..., None] * p)[..., :-1] + g_eal[..., None] * is_star
        grad = torch.zeros(B, S, V + 1, device=z.device)
        torch.mul(e, others[..., None] / s, out=grad[..., :V])
        grad.scatter_(-1, past, mine)
        grad = grad[..., :V].to(DTYPES[c.get("grad_dtype", c["dtype"])])
    return {"loss": loss, "terms": terms, "E_tv": E_tv, "E_eal": E_eal, "accept_tv": a_tv.flatten(),
            "accept_eal": a_eal.flatten(), "xstar": torch.where(has, star, -1).int().flatten(), "grad": grad}


def _count(c, B, S, device):
    """How many windows contain each row."""
    s = torch.arange(S, device=device)
    n = torch.minimum(s, torch.tensor(S - c["K"], device=device)) - (s - c["K"] + 1).clamp(min=0) + 1
    return n.clamp(min=0).float().expand(B, S)


def _history(c, rules, z):
    """Which entries each row's history holds, and how often its generated part does."""
    R, V = z.shape
    n = rules["hist_len"].long()
    row = torch.repeat_interleave(torch.arange(R, device=z.device), n)
    first = n.cumsum(0) - n
    place = torch.arange(row.numel(), device=z.device) - first[row]
    token = rules["tokens"][rules["hist_start"][row] + place].long()
    at = row * V + token
    seen = torch.zeros(R * V, dtype=torch.bool, device=z.device)
    seen[at] = True
    count = torch.zeros(R * V, device=z.device)
    count.index_add_(0, at, (place >= rules["prompt_len"][row]).float())
    return seen.view(R, V), count.view(R, V)


def _biased(rules, z):
    x = z.float()
    if "bias_ids" in rules:
        off = rules["bias_offsets"]
        row = torch.repeat_interleave(torch.arange(z.shape[0], device=z.device), off[1:] - off[:-1])
        x = x.index_put((row, rules["bias_ids"].long()), rules["bias_values"], accumulate=True)
    return x


def _blocked(rules, z):
    V = z.shape[1]
    v = torch.arange(V, device=z.device)
    m = rules["mask_row"].long()
    word = rules["mask"][m.clamp(min=0)][:, v >> 5]
    return (((word >> (v & 31).int()) & 1) == 0) & (m >= 0)[:, None]


def _plain_process(c, z, rules):
    x = _biased(rules, z)
    if "tokens" in rules:
        seen, count = _history(c, rules, z)
        rep = rules["repetition"][:, None]
        x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
        x -= rules["frequency"][:, None] * count + rules["presence"][:, None] * (count > 0)
    if "mask" in rules:
        x = torch.where(_blocked(rules, z), -math.inf, x)
    return x.to(z.dtype)


def _plain_process_bwd(c, z, grad, rules):
    g = grad.float()
    if "tokens" in rules:
        seen, _ = _history(c, rules, z)
        rep = rules["repetition"][:, None]
        g = torch.where(seen, torch.where(_biased(rules, z) > 0, g / rep, g * rep), g)
    if "mask" in rules:
        g = torch.where(_blocked(rules, z), 0.0, g)
    return g.to(grad.dtype)


# ----------------------------------------------------------------------- work
def work(case):
    c = case
    R, V, s = _rows(c), c["V"], BYTES[c["dtype"]]
    if c["op"] == "topk":
        # the logits once, the lists; a comparison, an exponential's argument and a sum for each entry
        return {"bytes": float(R * (V * s + c["k"] * (s + 4) + 4)), "flops": float(R * V * 4)}
    if c["op"] == "loss":
        sg = BYTES[c.get("grad_dtype", c["dtype"])] if c.get("grad", True) else 0
        return {"bytes": float(R * (V * (s + sg) + c["k"] * (s + 4) + 20)), "flops": float(R * V * 7)}
    # logits or gradients in and out, the contexts' tokens, the grammars and biases
    rules = c["N"] * c["hist"] * 4 + c["masks"] * (V // 8) + R * (36 if c["hist"] else 0) + R * c["bias"] * 4
    return {"bytes": float(R * V * 2 * s + rules), "flops": float(R * V)}


# -------------------------------------------------------------------- 64 bits
def _chunks(rows, V):
    n = max(1, (1 << 26) // V)
    return [(r, min(rows, r + n)) for r in range(0, rows, n)]


def _exact_topk(c, z):
    R, V, k, T = c["rows"], c["V"], c["k"], c["T"]
    ids = torch.empty(R, k, dtype=torch.int64, device=z.device)
    rest = torch.empty(R, dtype=torch.float64, device=z.device)
    for r0, r1 in _chunks(R, V):
        x = z[r0:r1].double()
        order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :k]
        ids[r0:r1] = order
        gone = torch.zeros_like(x, dtype=torch.bool).scatter_(1, order, True)
        rest[r0:r1] = torch.logsumexp(torch.where(gone, -math.inf, x / T), -1)
    return {"logits": z.double().gather(1, ids) if R * V < 1 << 28 else torch.stack(
        [z[r].double()[ids[r]] for r in range(R)]), "ids": ids.int(), "rest": rest}


def _exact_windows(a, c):
    """E of each window, and dE/da summed per row: by the definition, position by position."""
    K, (B, S) = c["K"], a.shape
    W = S - K + 1
    E = torch.zeros(B, W, dtype=torch.float64, device=a.device)
    d = torch.zeros_like(a)
    for j in range(K):
        up_to = torch.ones(B, W, dtype=torch.float64, device=a.device)
        for i in range(j):
            up_to = up_to * a[:, i:i + W]
        E += up_to * a[:, j:j + W]
        tail = torch.ones_like(up_to)
        run_ = torch.ones_like(up_to)
        for i in range(j + 1, K):
            run_ = run_ * a[:, i:i + W]
            tail = tail + run_
        d[:, j:j + W] += up_to * tail
    return E.flatten(), d


def _exact_loss(c, z, top, ids, rest):
    B, S, V = z.shape
    R = B * S
    w = WEIGHTS[c["weights"]]
    z, top, ids = z.view(R, V), top.view(R, -1).double(), ids.view(R, -1).long()
    valid = (ids >= 0) & (ids < V) & (top > -math.inf)
    t = torch.where(valid, top / c["tt"], -math.inf)
    tr = torch.full((R,), -math.inf, dtype=torch.float64, device=z.device) if rest is None else rest.view(R).double()
    norm = torch.logsumexp(torch.cat([t, tr[:, None]], 1), 1)
    empty = norm == -math.inf
    norm = torch.where(empty, 0.0, norm)
    p, pr = (t - norm[:, None]).exp(), (tr - norm).exp()
    at = torch.where(valid, ids, 0)
    logq, logqr = torch.empty_like(t), torch.full_like(tr, -math.inf)
    for r0, r1 in _chunks(R, V):
        lq = torch.log_softmax(z[r0:r1].double() / c["td"], -1)
        logq[r0:r1] = lq.gather(1, at[r0:r1])
        if rest is not None:
            row = torch.arange(r1 - r0, device=z.device)[:, None].expand_as(at[r0:r1])
            keep = valid[r0:r1]
            lq[row[keep], at[r0:r1][keep]] = -math.inf
            logqr[r0:r1] = torch.logsumexp(lq, 1)
    q, qr = torch.where(valid, logq.exp(), 0.0), logqr.exp()
    kl = torch.where(p > 0, p * (t - norm[:, None] - logq), 0.0).sum(1)
    kl += torch.where(pr > 0, pr * (tr - norm - logqr), 0.0)
    a_tv = torch.minimum(p, q).sum(1) + torch.minimum(pr, qr)
    below, below_r = (q < p).double(), (qr < pr).double()
    qlt = (q * below).sum(1) + qr * below_r
    best = torch.where(valid, top, -math.inf).amax(1, keepdim=True)
    star = torch.where(valid & (top == best), ids, V).amin(1)
    star = torch.where(star < V, star, -1)
    hit = valid & (ids == star[:, None])
    a_eal = torch.where(hit, q, 0.0).sum(1)
    E_tv, d_tv = _exact_windows(a_tv.view(B, S), c)
    E_eal, d_eal = _exact_windows(a_eal.view(B, S), c)
    W = E_tv.numel()
    inside = torch.zeros(B, S, dtype=torch.float64, device=z.device)
    for j in range(c["K"]):
        inside[:, j:j + S - c["K"] + 1] += 1
    terms = [-E_tv.mean() if w[0] else 0.0, -E_eal.mean() if w[1] else 0.0, kl.mean() if w[2] else 0.0,
             (inside.view(R) * (1 - a_tv)).sum() / (W * c["K"]) if w[3] else 0.0]
    grad = None
    if c.get("grad", True):
        grad = torch.empty(R, V, dtype=torch.float64, device=z.device)
        c_tv = (-w[0] * d_tv - w[3] * inside / c["K"]).view(R, 1) / W
        c_eal = -w[1] * d_eal.view(R, 1) / W * a_eal[:, None]
        c_kl = torch.where(empty, 0.0, w[2] / R)[:, None]
        mine = q * (c_tv * (below - qlt[:, None]) - c_eal + c_kl) - c_kl * p + c_eal * hit
        share = torch.where(qr > 0, pr / qr, 0.0)[:, None]
        for r0, r1 in _chunks(R, V):
            s = slice(r0, r1)
            g = torch.softmax(z[s].double() / c["td"], -1)
            g *= c_tv[s] * (below_r[s, None] - qlt[s, None]) - c_eal[s] + c_kl[s] * (1 - share[s])
            row = torch.arange(r1 - r0, device=z.device)[:, None].expand_as(at[s])
            g[row[valid[s]], at[s][valid[s]]] = mine[s][valid[s]]
            grad[s] = g / c["td"]
        grad = grad.view(B, S, V)
    terms = torch.tensor([float(x) for x in terms], dtype=torch.float64)
    return {"loss": (terms * torch.tensor(w, dtype=torch.float64)).sum().reshape(1), "terms": terms, "E_tv": E_tv,
            "E_eal": E_eal, "accept_tv": a_tv, "accept_eal": a_eal, "xstar": star.int(), "grad": grad}


def _exact_process(c, z, rules, grad=None):
    """Both directions, a block of rows at a time, from dense tables of what the rules say of a row."""
    R, V = z.shape
    dev = z.device
    out = torch.empty(R, V, dtype=torch.float64, device=dev)
    if "tokens" in rules:
        lens, starts, prompts = (rules[n].tolist() for n in ("hist_len", "hist_start", "prompt_len"))
    offsets = rules["bias_offsets"].tolist() if "bias_ids" in rules else None
    which = rules["mask_row"].tolist() if "mask" in rules else None
    shift = torch.arange(32, device=dev)
    for r in range(R):
        x = z[r].double()
        if offsets is not None:
            b = slice(offsets[r], offsets[r + 1])
            x[rules["bias_ids"][b].long()] += rules["bias_values"][b].double()
        y = x if grad is None else grad[r].double()
        if "tokens" in rules:
            words = rules["tokens"][starts[r]:starts[r] + lens[r]].long()
            times = torch.bincount(words[prompts[r]:], minlength=V).double()
            seen = torch.bincount(words, minlength=V) > 0
            rep = rules["repetition"][r].double()
            y = torch.where(seen, torch.where(x > 0, y / rep, y * rep), y)
            if grad is None:
                y = y - rules["frequency"][r].double() * times - rules["presence"][r].double() * (times > 0)
        if which is not None and which[r] >= 0:
            free = (rules["mask"][which[r]][:, None] >> shift & 1).flatten()[:V] != 0
            y = torch.where(free, y, -math.inf if grad is None else 0.0)
        out[r] = y
    return out


def exact(case, seed):
    c = case
    if c["op"].startswith("process") and _rows(c) > 20000:
        return None  # a row at a time: too slow
    zd, zt = _logits(c, seed)
    if c["op"] == "topk":
        return _exact_topk(c, zt)
    if c["op"] == "loss":
        top, ids, rest = _lists(c, zt, seed)
        lead = (c["B"], c["S"])
        del zt
        return _exact_loss(c, zd.view(*lead, -1), top, ids, rest)
    st = prepare(c, seed)
    return _exact_process(c, st["z"], st["rules"], st.get("grad"))
