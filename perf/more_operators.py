"""The measured cases of the operators on logits [B, rows, V] next to the tree path: penalties, biases and grammar masks
(adjust_logits), the target's choice along a draft tree (verify_tree), and the drafter's distillation from a teacher's top
logits (distill, distill_grad), over the range of batches, vocabularies, histories and types that serving and training use.

A case is a dict of plain values:

op       "adjust" (adjust_logits), "verify" (verify_tree), "distill" (loss and gradient in one call), "loss" (distill without
         a gradient) or "grad" (distill_grad, from the sums that an earlier loss call kept)
dtype    "bf16", "f16" or "f32" logits
B, T, V  sequences, rows of a sequence (block positions; in a tree 1 + cap: the root and the nodes), vocabulary
ragged   lengths differ over the batch, zero and one among them where there are enough sequences; else all are full
tree     the rows are a draft tree's: "adjust" counts the tokens on a row's path too
H        tokens of a sequence's history at most
penalty  repetition, presence and frequency penalties by sequence
N        biased tokens of a sequence, padding among them
grammar  "" (none), "few" (a handful of tokens is allowed), "most" (a few are forbidden) or "shared" (one mask for all rows)
K        tokens that the teacher lists
tail     the teacher lists log-probabilities, what they leave is the rest's; else logits, renormalised over the list
tau      temperature
masked   part of the rows that carry no weight
pad      elements between the end of a row and the next one's start
"""

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
PATH = 17                      # rows of a path at most: the root and 16 nodes
LARGEST = 1024 * 151936        # logits of the largest listed case of "adjust" and "distill" in 16 bits


def _case(name, **kw):
    c = dict(op="adjust", dtype="bf16", B=1, T=1, V=151936, ragged=False, tree=False, H=0, penalty=False, N=0, grammar="",
             K=0, tail=False, tau=1.0, masked=0.0, pad=0)
    c.update(kw)
    c["name"] = name
    return c


def listed():
    return [
        # the next token of one request with penalties: latency counts
        _case("adjust_one", H=700, penalty=True),
        # the next token of a serving batch: penalties, biases, and a grammar each
        _case("adjust_decode_64", B=64, H=8192, ragged=True, penalty=True, N=300, grammar="few"),
        # a batch of the drafter's blocks before their trees are built
        _case("adjust_blocks_64", B=64, T=16, H=2048, ragged=True, penalty=True, N=32),
        # the target's logits at the nodes of a few draft trees, of a vocabulary whose rows start anywhere
        _case("adjust_trees_8", dtype="f32", B=8, T=129, V=100003, tree=True, ragged=True, H=4096, penalty=True, grammar="most"),
        # one request's tree is verified: latency counts
        _case("verify_one", op="verify", T=65, tree=True),
        # a serving batch's trees are verified
        _case("verify_32", op="verify", B=32, T=257, tree=True, ragged=True),
        # small trees over fp32 logits of odd length, an empty one among them
        _case("verify_odd", op="verify", dtype="f32", B=7, T=33, V=100003, tree=True, ragged=True),
        # a few rounds of a drafter that learns while it serves
        _case("distill_online", op="distill", B=4, T=16, K=8),
        # a training step of the drafter
        _case("distill_train", op="distill", B=64, T=16, K=8, tau=1.5, masked=0.1),
        # ... from log-probabilities with the rest's mass, in fp32, rows of odd length
        _case("distill_tail", op="distill", dtype="f32", B=24, T=15, V=100003, K=16, tail=True, masked=0.2),
        # the loss alone, on held-out text
        _case("loss_eval", op="loss", B=128, T=16, K=16, tail=True, masked=0.05),
        # the backward pass by itself, from a long list
        _case("grad_long_list", op="grad", dtype="f16", B=40, T=13, V=65537, K=128, tau=2.0, masked=0.3, pad=7),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    """One more case of the same ranges; its cost is bounded by the largest listed ones'."""
    c = _case("")
    del c["name"]
    c["op"] = rng.choice(["adjust", "adjust", "verify", "distill", "distill", "loss", "grad"])
    c["dtype"] = rng.choice(["bf16", "bf16", "f16", "f32"])
    c["V"] = rng.choice([_log_int(rng, 1000, 151936), rng.choice([151936, 100003, 65537, 32000, 1024])])
    c["pad"] = rng.choice([0, 0, 0, 1, 8, 13])
    most = LARGEST * 2 // SIZE[c["dtype"]] // c["V"]           # rows
    if c["op"] == "verify":
        c["tree"], c["ragged"] = True, rng.random() < 0.6
        c["T"] = 1 + _log_int(rng, 1, 512)
        c["B"] = max(1, min(_log_int(rng, 1, 64), 32 * 257 * 151936 * 2 // SIZE[c["dtype"]] // c["V"] // c["T"]))
    elif c["op"] == "adjust":
        c["tree"], c["ragged"] = rng.random() < 0.4, rng.random() < 0.6
        c["T"] = 1 + _log_int(rng, 1, 256) if c["tree"] else rng.choice([1, 1, _log_int(rng, 1, 32)])
        c["B"] = max(1, min(_log_int(rng, 1, 256), most // c["T"]))
        c["penalty"] = rng.random() < 0.75
        c["H"] = _log_int(rng, 1, 16384) if c["penalty"] else 0
        c["N"] = rng.choice([0, 0, 1, _log_int(rng, 1, 1024)])
        c["grammar"] = rng.choice(["", "", "few", "most", "shared"])
    else:
        rows = _log_int(rng, 1, most)
        c["T"] = rng.choice([1, 7, 15, 16, 16, 32])
        c["B"] = max(1, min(rows, most) // c["T"])
        c["K"] = rng.choice([1, 4, 8, 8, 16, 16, _log_int(rng, 1, 256)])
        c["tail"] = rng.random() < 0.5
        c["tau"] = 1.0 if c["tail"] else rng.choice([1.0, 1.0, round(math.exp(rng.uniform(-1.0, 1.5)), 3)])
        c["masked"] = rng.choice([0.0, 0.0, round(rng.uniform(0.0, 0.6), 2)])
    return c


# ---------------------------------------------------------------- sizes that follow from a case alone

def _spread(n, most, ragged):
    """`n` lengths up to `most`: full ones, or spread over [0, 1] of it with an empty and a one-token one."""
    if not ragged:
        return [most] * n
    part = (1.0, 0.53, 0.77, 0.0, 0.35, 0.911, 0.66)
    got = [int(most * part[b % 7]) for b in range(n)]
    if n >= 5:
        got[4] = min(1, most)
    return got


def _trees(c):
    """For each sequence: its nodes, all cap parents in breadth-first order (-1: the root), and the path that the target
    takes, as rows (0: the root, i: node i - 1)."""
    cap = c["T"] - 1
    got = []
    for b, n in enumerate(_spread(c["B"], cap, c["ragged"])):
        r = 0.2 + 0.4 * ((b + 1) * 0.6180339887498949 % 1.0)
        parent = [min(int(i * r), i) - 1 for i in range(cap)]
        row, path = n, []
        while row > 0:
            path.append(row)
            row = parent[row - 1] + 1
        path = [0] + path[::-1]
        got.append((n, parent, path[:1 + (3 + 5 * b) % len(path)]))
    return got


def _masked(c):
    """How many rows carry no weight."""
    return int(c["masked"] * c["B"] * c["T"])


def _rows(c):
    if c["tree"]:
        return sum(n + 1 for n, _, _ in _trees(c))
    return c["B"] * c["T"]


def work(c):
    V, e = c["V"], SIZE[c["dtype"]]
    if c["op"] == "verify":
        trees = _trees(c)
        steps = sum(len(path) for _, _, path in trees)
        nodes = sum(n for n, _, _ in trees)
        return {"bytes": steps * V * e + nodes * 8 + c["B"] * (PATH * 8 + 8) + c["B"] * c["T"] * 4, "flops": steps * V}
    if c["op"] == "adjust":
        rows = _rows(c)
        words = (V + 31) // 32 * (c["B"] if c["grammar"] == "shared" else rows if c["grammar"] else 0)
        history = sum(_spread(c["B"], c["H"], c["ragged"]))
        return {"bytes": rows * V * 2 * e + words * 4 + history * 4 + c["B"] * (c["N"] * 8 + 12), "flops": rows * V}
    rows = c["B"] * c["T"]
    live = rows - _masked(c)
    read = live * (V * e + c["K"] * 8)
    written = 0 if c["op"] == "loss" else rows * V * e
    return {"bytes": read + written + rows * 16, "flops": live * V * (4 if c["op"] == "loss" else 8)}


# ---------------------------------------------------------------- the plain form

def _plain_path_counts(c, s):
    """[B, T, V] how often each token stands on each row's path."""
    B, T, V = c["B"], c["T"], c["V"]
    got = torch.zeros((B, T, V), device="cuda")
    node = torch.arange(T, device="cuda").expand(B, -1) - 1                        # (row 0 has none)
    live = torch.arange(T, device="cuda") <= s["count"][:, None]
    for _ in range(T):
        on = live & (node >= 0)
        if not bool(on.any()):
            break
        at = node.clamp(min=0)
        tok = s["token_ids"].to(torch.int64).gather(1, at)
        got.scatter_add_(2, tok[..., None], on[..., None].float())
        node = torch.where(on, s["parent"].to(torch.int64).gather(1, at), -1)
    return got


def _plain_adjust(c, s):
    B, T, V = c["B"], c["T"], c["V"]
    x = s["logits"].float()
    if c["penalty"]:
        tok = s["history"].to(torch.int64)
        there = torch.arange(c["H"], device="cuda") < s["history_len"][:, None]
        there = there & (tok >= 0) & (tok < V)
        count = torch.zeros((B, V), device="cuda").scatter_add_(1, tok.clamp(0, V - 1), there.float())[:, None]
        if c["tree"]:
            count = count + _plain_path_counts(c, s)
        part = lambda name: s[name][:, None, None]
        less = torch.where(x > 0, x / part("repetition"), x * part("repetition")) - part("frequency") * count - part("presence")
        x = torch.where(count > 0, less, x)
    if c["N"]:
        t = s["bias_ids"].to(torch.int64)
        t = torch.where((t >= 0) & (t < V), t, V)
        place = torch.arange(1, c["N"] + 1, device="cuda").expand(B, -1)
        last = torch.zeros((B, V + 1), dtype=torch.int64, device="cuda").scatter_reduce_(1, t, place, "amax")[:, :V]
        bias = torch.nn.functional.pad(s["bias"], (1, 0)).gather(1, last)          # (of a token listed twice the last)
        x = x + bias[:, None]
    if c["grammar"]:
        bits = (s["allowed"][..., None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        x = torch.where(bits.flatten(-2)[..., :V] != 0, x, -math.inf)
    if c["tree"]:
        live = torch.arange(T, device="cuda") <= s["count"][:, None]
        return torch.where(live[..., None], x.to(TYPES[c["dtype"]]), s["out"])
    return x.to(TYPES[c["dtype"]])


def _plain_verify(c, s):
    B, T = c["B"], c["T"]
    x = s["logits"].float()
    x = torch.where(torch.isnan(x), -math.inf, x)
    chosen = x.argmax(-1)                                                          # [B, T] (the first of equals)
    chosen = torch.where(x.amax(-1) > -math.inf, chosen, -1)
    nodes = torch.arange(T - 1, device="cuda")
    live = nodes < s["count"][:, None]
    row = torch.zeros(B, dtype=torch.int64, device="cuda")
    going = torch.ones(B, dtype=torch.bool, device="cuda")
    accepted = torch.zeros(B, dtype=torch.int32, device="cuda")
    weight = torch.zeros((B, T), device="cuda")
    index, tokens = [], []
    for _ in range(PATH):
        t = chosen.gather(1, row[:, None])[:, 0]
        index.append(torch.where(going, row, -1))
        tokens.append(torch.where(going, t, -1))
        weight.scatter_add_(1, row[:, None], going[:, None].float())
        accepted += going
        hit = live & (s["parent"] == row[:, None] - 1) & (s["token_ids"] == t[:, None])
        first = torch.where(hit, nodes, T).amin(1)
        going = going & (first < T)
        row = torch.where(going, first + 1, row)
    return accepted, torch.stack(index, 1).to(torch.int32), torch.stack(tokens, 1).to(torch.int32), weight


def _plain_teacher(c, s):
    """The teacher's probabilities [B, T, K], their logarithms, and the rest's probability [B, T]."""
    t = s["target"]
    if c["tail"]:
        p = t.exp()
        return p, t, (1.0 - p.sum(-1)).clamp(min=0.0)
    t = t / c["tau"]
    t = t - t.amax(-1, keepdim=True)
    logp = t - t.exp().sum(-1, keepdim=True).log()
    return logp.exp(), logp, torch.zeros_like(t[..., 0])


def _plain_student(c, s):
    """The student's log-probabilities [B, T, V], which tokens are listed, log(1 - Q) [B, T], and the largest logit of a
    row with the sum of the exponentials of the distances to it [B, T, 2]."""
    x = s["logits"].float()
    top = x.amax(-1, keepdim=True)
    x = (x - top) / c["tau"]
    e = x.exp()
    total = e.sum(-1, keepdim=True)
    on = torch.zeros(x.shape, dtype=torch.bool, device="cuda").scatter_(2, s["ids"].to(torch.int64), True)
    rest = torch.where(on, 0.0, e).sum(-1)
    return x - total.log(), on, rest.log() - total.log()[..., 0], torch.cat((top, total), -1)


def _plain_distill(c, s):
    p, logp, rho = _plain_teacher(c, s)
    logq, on, log_rest, stats = _plain_student(c, s)
    ids, w = s["ids"].to(torch.int64), s["weight"]
    out = []
    if c["op"] != "grad":
        loss = (p * (logp - logq.gather(2, ids))).sum(-1)
        if c["tail"]:
            loss = loss + torch.where(rho > 0, rho * (rho.log() - log_rest), 0.0)
        out += [torch.where(w != 0, loss * w, 0.0), torch.where(w[..., None] != 0, stats, 0.0)]
    if c["op"] != "loss":
        q = logq.exp()
        mass = (p.sum(-1) + rho)[..., None]
        g = q * torch.where(on, mass, mass - (rho / log_rest.exp())[..., None])
        g = g.scatter_add(2, ids, -p) * (w / c["tau"])[..., None]
        out.append(torch.where(w[..., None] != 0, g, 0.0).to(TYPES[c["dtype"]]))
    return tuple(out)


# ---------------------------------------------------------------- inputs

def _logits(c, gen, rows):
    """[rows, T, V] logits with a few tokens far above the others, in rows that lie V + pad elements apart."""
    x = torch.randn((rows, c["T"], c["V"] + c["pad"]), generator=gen, device="cuda")
    x = 2.0 * x + 6.0 * (x > 3.0)
    return x.to(TYPES[c["dtype"]])


def _all_logits(c, gen):
    if c["op"] == "verify":                                                        # (large: one sequence at a time)
        x = torch.empty((c["B"], c["T"], c["V"] + c["pad"]), dtype=TYPES[c["dtype"]], device="cuda")
        for b in range(c["B"]):
            x[b] = _logits(c, gen, 1)[0]
    else:
        x = _logits(c, gen, c["B"])
    return x[..., :c["V"]]


def _grammar(c, gen):
    B, T, V, words = c["B"], c["T"], c["V"], (c["V"] + 31) // 32
    shape = (B, 1 if c["grammar"] == "shared" else T, words)
    if c["grammar"] != "shared":
        bits = torch.empty(shape, dtype=torch.int32, device="cuda")
        for b in range(B):
            named = torch.zeros((T, words * 32), dtype=torch.bool, device="cuda")
            named.scatter_(1, torch.randint(V, (T, 24 if c["grammar"] == "few" else 200), generator=gen, device="cuda"), True)
            word = (named.view(T, words, 32).to(torch.int64) << torch.arange(32, device="cuda")).sum(-1)
            bits[b] = torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32)
        return bits if c["grammar"] == "few" else ~bits
    bits = torch.randint(-2 ** 31, 2 ** 31, shape, generator=gen, device="cuda").to(torch.int32)
    off = torch.rand((*shape[:2], (words + 63) // 64), generator=gen, device="cuda") < 0.5     # whole stretches at once
    bits = torch.where(off.repeat_interleave(64, 2)[..., :words], 0, bits)
    return bits.expand(-1, T, -1)


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    B, T, V = c["B"], c["T"], c["V"]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    rand = lambda *shape: torch.rand(shape, generator=gen, device="cuda")
    s = {"case": c, "logits": _all_logits(c, gen)}
    if c["tree"]:
        trees = _trees(c)
        s["count"] = i32([n for n, _, _ in trees])
        s["parent"] = i32([parent for _, parent, _ in trees]).view(B, T - 1)
        s["token_ids"] = torch.randint(V, (B, T - 1), generator=gen, device="cuda", dtype=torch.int32)
    if c["op"] == "verify":
        for b, (n, parent, path) in enumerate(trees):                              # the target agrees up to the path's end
            for row, after in zip(path, path[1:] + [0]):
                t = s["token_ids"][b, after - 1] if after else (s["token_ids"][b, T - 2] + 1) % V
                s["logits"][b, row].index_fill_(0, t.to(torch.int64), 60.0)
        s["accepted"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        s["index"] = torch.zeros((B, PATH), dtype=torch.int32, device="cuda")
        s["tokens"] = torch.zeros((B, PATH), dtype=torch.int32, device="cuda")
        s["weight"] = torch.zeros((B, T), device="cuda")
        if own:
            from paper_2606_01813_amd import verify_workspace
            s["workspace"] = verify_workspace(s["logits"])
        return s
    if c["op"] == "adjust":
        if c["penalty"]:
            # text repeats itself: few tokens make up most of it, and there is padding
            tok = (V * rand(B, c["H"]) ** 6).to(torch.int32).clamp(max=V - 1)
            s["history"] = torch.where(rand(B, c["H"]) < 0.02, -1, tok)
            s["history_len"] = i32(_spread(B, c["H"], c["ragged"]))
            s["repetition"] = 1.0 + 0.3 * rand(B)
            s["presence"], s["frequency"] = rand(B), 0.5 * rand(B)
        if c["N"]:
            ids = torch.randint(V, (B, c["N"]), generator=gen, device="cuda", dtype=torch.int32)
            s["bias_ids"] = torch.where(rand(B, c["N"]) < 0.1, -1, ids)
            s["bias"] = 20.0 * rand(B, c["N"]) - 10.0
        if c["grammar"]:
            s["allowed"] = _grammar(c, gen)
        s["out"] = torch.zeros((B, T, V), dtype=TYPES[c["dtype"]], device="cuda")
        return s
    # the teacher: the largest of the same logits with noise, so that it agrees with the student as a teacher does
    lse = torch.empty((B, T), device="cuda")
    ids = torch.empty((B, T, c["K"]), dtype=torch.int32, device="cuda")
    top = torch.empty((B, T, c["K"]), device="cuda")
    for b in range(0, B, 8):
        x = s["logits"][b:b + 8].float()
        x = x + torch.randn(x.shape, generator=gen, device="cuda")
        best = x.topk(c["K"], dim=-1)
        m = best.values[..., :1]
        lse[b:b + 8] = m[..., 0] + (x - m).exp().sum(-1).log()
        ids[b:b + 8], top[b:b + 8] = best.indices.to(torch.int32), best.values
    s["ids"] = ids
    s["target"] = top - lse[..., None] if c["tail"] else top
    w = (0.5 + rand(B, T)) / (1 if c["dtype"] == "f16" else B * T)                 # (f16 trains with a scaled loss)
    off = rand(B * T).argsort()[:_masked(c)]
    w.view(-1)[off] = 0.0
    s["weight"] = w
    s["loss"] = torch.zeros((B, T), device="cuda")
    s["stats"] = torch.zeros((B, T, 2), device="cuda")
    if c["op"] == "grad":
        for b in range(0, B, 8):
            x = s["logits"][b:b + 8].double()
            m = x.amax(-1)
            s["stats"][b:b + 8, :, 0] = m
            s["stats"][b:b + 8, :, 1] = ((x - m[..., None]) / c["tau"]).exp().sum(-1)
    if c["op"] != "loss":
        s["grad"] = torch.zeros((B, T, V + c["pad"]), dtype=TYPES[c["dtype"]], device="cuda")[..., :V]
    if own:
        from paper_2606_01813_amd import distill, distill_workspace
        s["workspace"] = distill_workspace(s["logits"])
        s["kept"] = torch.zeros((B, T, 3), device="cuda")                          # as the calls have them: with the rest's sum
        if c["op"] == "grad":
            distill(s["logits"], s["ids"], s["target"], s["loss"], stats=s["kept"], weight=w, temperature=c["tau"], tail=c["tail"],
                    workspace=s["workspace"])
    return s


def run(s):
    c = s["case"]
    if not own:
        with torch.no_grad():
            return (_plain_adjust if c["op"] == "adjust" else _plain_verify if c["op"] == "verify" else _plain_distill)(c, s)
    from paper_2606_01813_amd import adjust_logits, distill, distill_grad, verify_tree
    if c["op"] == "adjust":
        names = ("history", "history_len", "repetition", "presence", "frequency", "bias_ids", "bias", "allowed", "token_ids",
                 "parent", "count")
        return adjust_logits(s["logits"], s["out"], **{n: s[n] for n in names if n in s})
    if c["op"] == "verify":
        verify_tree(s["logits"], s["token_ids"], s["parent"], s["count"], s["accepted"], s["index"], s["tokens"],
                    weight=s["weight"], workspace=s["workspace"])
        return s["accepted"], s["index"], s["tokens"], s["weight"]
    how = dict(weight=s["weight"], temperature=c["tau"], tail=c["tail"], workspace=s["workspace"])
    if c["op"] == "grad":
        return (distill_grad(s["logits"], s["ids"], s["target"], s["kept"], s["grad"], **how),)
    distill(s["logits"], s["ids"], s["target"], s["loss"], stats=s["kept"], grad=s.get("grad"), **how)
    stats = s["kept"][..., :2]
    return (s["loss"], stats) if c["op"] == "loss" else (s["loss"], stats, s["grad"])


# ---------------------------------------------------------------- the definition in 64 bits

def _exact_adjust(c, s):
    V, out = c["V"], s["out"].double()
    for b in range(c["B"]):
        n = int(s["count"][b]) + 1 if c["tree"] else c["T"]
        x = s["logits"][b, :n].double()
        if c["penalty"]:
            h = s["history"][b, :int(s["history_len"][b])].to(torch.int64)
            base = torch.bincount(h[(h >= 0) & (h < V)], minlength=V)
            rep, pres, freq = (float(s[k][b]) for k in ("repetition", "presence", "frequency"))
            tok, par = (s[k][b].tolist() for k in ("token_ids", "parent")) if c["tree"] else (None, None)
            for i in range(n):
                count = base.clone() if c["tree"] else base
                node = i - 1 if c["tree"] else -1
                while node >= 0:
                    count[tok[node]] += 1
                    node = par[node]
                at = count.nonzero()[:, 0]
                y = x[i, at]
                y = torch.where(y > 0, y / rep, y * rep)
                x[i, at] = y - freq * count[at].double() - pres
        if c["N"]:
            last = {t: v for t, v in zip(s["bias_ids"][b].tolist(), s["bias"][b].tolist()) if 0 <= t < V}
            if last:
                x[:, torch.tensor(list(last), device="cuda")] += torch.tensor(list(last.values()), dtype=torch.float64, device="cuda")
        if c["grammar"]:
            v = torch.arange(V, device="cuda")
            for i in range(n):
                bit = (s["allowed"][b, i].to(torch.int64)[v // 32] >> (v % 32)) % 2
                x[i, bit == 0] = -math.inf
        out[b, :n] = x
    return out


def _exact_verify(c, s):
    B, T = c["B"], c["T"]
    accepted = torch.zeros(B, dtype=torch.int32, device="cuda")
    index = torch.full((B, PATH), -1, dtype=torch.int32, device="cuda")
    tokens = torch.full((B, PATH), -1, dtype=torch.int32, device="cuda")
    weight = torch.zeros((B, T), dtype=torch.float64, device="cuda")
    for b in range(B):
        n, tok, par = int(s["count"][b]), s["token_ids"][b].tolist(), s["parent"][b].tolist()
        row = 0
        for step in range(PATH):
            x = s["logits"][b, row].double().nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf)
            top = float(x.max())
            t = int((x == top).nonzero()[0, 0]) if top > -math.inf else -1
            index[b, step], tokens[b, step], accepted[b], weight[b, row] = row, t, step + 1, 1.0
            child = [i for i in range(n) if par[i] == row - 1 and tok[i] == t]
            if not child:
                break
            row = child[0] + 1
    return accepted, index, tokens, weight


def _exact_distill(c, s):
    B, T = c["B"], c["T"]
    loss = torch.zeros((B, T), dtype=torch.float64, device="cuda")
    norm = torch.zeros((B, T, 2), dtype=torch.float64, device="cuda")
    grad = torch.zeros((B, T, c["V"]), dtype=torch.float64, device="cuda") if c["op"] != "loss" else None
    for b in range(B):
        x = s["logits"][b].double() / c["tau"]
        ids, w = s["ids"][b].to(torch.int64), s["weight"][b].double()
        t = s["target"][b].double()
        top = x.max(1, keepdim=True).values
        e = torch.exp(x - top)
        lse = top[:, 0] + torch.log(e.sum(1))
        p = torch.exp(t) if c["tail"] else torch.softmax(t / c["tau"], 1)
        rho = (1.0 - p.sum(1)).clamp(min=0.0) if c["tail"] else torch.zeros_like(lse)
        full = torch.zeros_like(x).scatter_add_(1, ids, p)
        on = full.new_zeros(x.shape).scatter_(1, ids, 1.0)
        rest = (e * (1.0 - on)).sum(1)                                             # (of what the row's largest is 1 of)
        logp = t if c["tail"] else torch.log(p)
        one = (p * (logp - (x.gather(1, ids) - lse[:, None]))).sum(1)
        some = rho > 0
        one[some] += rho[some] * (torch.log(rho[some]) - (top[some, 0] + torch.log(rest[some]) - lse[some]))
        loss[b] = torch.where(w != 0, w * one, 0.0)
        norm[b] = torch.where(w[:, None] != 0, torch.stack((top[:, 0] * c["tau"], e.sum(1)), 1), 0.0)
        if grad is not None:
            q = torch.exp(x - lse[:, None])
            teacher = full + torch.where(some[:, None], rho[:, None] * (1.0 - on) * e / rest[:, None], 0.0)
            grad[b] = torch.where(w[:, None] != 0, w[:, None] / c["tau"] * (q * (p.sum(1) + rho)[:, None] - teacher), 0.0)
    return {"loss": (loss, norm), "grad": (grad,), "distill": (loss, norm, grad)}[c["op"]]


def exact(c, seed):
    if c["op"] == "adjust" and c["tree"] and _rows(c) > 4000:                      # (row by row: too long)
        return None
    s = prepare(c, seed)
    return (_exact_adjust if c["op"] == "adjust" else _exact_verify if c["op"] == "verify" else _exact_distill)(c, s)
