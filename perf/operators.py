"""The operators beside the scoring step, as they are measured: products with 4-bit weights and group scales that give whole rows
of logits, the draw of the next word from them, and the loss against a teacher's top logits with its gradient.

`own` false: elementary torch operations; true: the calls a user makes of paper_2007_11794_amd.  Both take what prepare() gives.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------------------------------ cases
def listed():
    def q4(name, B, V, H, group, x, y, scale, zero):
        return {"name": name, "op": "q4", "B": B, "V": V, "H": H, "group": group, "x": x, "y": y, "scale": scale, "zero": zero}

    def sample(name, N, V, dtype, rule):
        return {"name": name, "op": "sample", "N": N, "V": V, "dtype": dtype, "rule": rule}

    def distill(name, part, N, V, K, dtype, T, label):
        return {"name": name, "op": "distill", "part": part, "N": N, "V": V, "K": K, "dtype": dtype, "T": T, "label": label}

    return [
        # the tiny workload's vocabulary and hidden size, one history: a call that is all latency
        q4("q4 tiny, 1 row", 1, 1000, 64, 32, "f32", "f32", "f32", False),
        # one sentence being written with the large-vocabulary model
        q4("q4 large vocabulary, 1 row", 1, 65536, 512, 128, "f32", "f32", "bf16", False),
        # sixteen sentences at once with the stress model, in bf16 throughout, weights with zero points
        q4("q4 stress, 16 rows, bf16", 16, 200000, 1024, 64, "bf16", "bf16", "bf16", True),
        # the paper's own regime: a million words, a hidden layer of 100 units (rows of 50 bytes), a few histories
        q4("q4 million words, 8 rows", 8, 1000000, 100, 32, "f32", "f32", "f32", False),
        # a batch of histories with the wsj-sized model: rows enough to fill matrix tiles, an odd number of them
        q4("q4 wsj, 61 rows", 61, 20000, 256, 32, "f32", "f32", "f32", True),
        # the next word of one sentence, the usual limits
        sample("sample 1 row, top-k and top-p", 1, 65536, "f32", "both"),
        # a text generator's batch, each row with limits of its own
        sample("sample 256 rows, mixed", 256, 65536, "f32", "mixed"),
        # few sentences over a million words in bf16, where many words tie, top-p alone: the long tail is summed too
        sample("sample 16 rows, million words", 16, 1000000, "bf16", "top_p"),
        # a handful of frames through the tiny model: the loss alone, as in a held-out check
        distill("distill loss, 8 rows", "loss", 8, 1000, 16, "f32", 2.0, False),
        # a training batch of the large-vocabulary student in bf16, soft targets and labels, loss and gradient at once
        distill("distill step, bf16 with labels", "step", 1024, 65536, 64, "bf16", 2.0, True),
        # rows too long for one workgroup's registers, fp32
        distill("distill step, long rows", "step", 256, 200000, 100, "f32", 1.0, False),
        # gradient alone, from kept statistics, at an odd vocabulary
        distill("distill backward, odd rows", "backward", 509, 20011, 33, "f32", 3.0, True),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["q4", "sample", "distill"])
    if op == "q4":
        x = rng.choice(["f32", "bf16"])
        c = {"op": op, "B": _spread(rng, 1, 64), "V": _spread(rng, 600, 300000), "H": _spread(rng, 32, 1024), "group": rng.choice([32, 64, 128]),
             "x": x, "y": rng.choice(["f32", "bf16"]) if x == "bf16" else "f32", "scale": rng.choice(["f32", "bf16"]), "zero": rng.random() < 0.5}
        while c["V"] * c["H"] > 200000 * 1024 or c["V"] * c["B"] > 8000000:
            c["V"] = max(600, c["V"] // 2 - 1)
        return c
    if op == "sample":
        c = {"op": op, "N": _spread(rng, 1, 256), "V": _spread(rng, 600, 300000), "dtype": rng.choice(["f32", "bf16"]),
             "rule": rng.choice(["both", "top_p", "top_k", "min_p", "none", "mixed"])}
        while c["N"] * c["V"] > 16000000:
            c["V"] = c["V"] // 2 - 1
        return c
    c = {"op": op, "part": rng.choice(["loss", "step", "backward"]), "N": _spread(rng, 1, 2048), "V": _spread(rng, 600, 200000), "K": _spread(rng, 1, 256),
         "dtype": rng.choice(["f32", "bf16"]), "T": rng.choice([1.0, 1.5, 2.0, 4.0]), "label": rng.random() < 0.5}
    while c["N"] * c["V"] > 50000000:
        c["V"] = c["V"] // 2 - 1
    return c


# ----------------------------------------------------------------------------------------------------------------- inputs
def _logits(g, N, V, dtype):
    """Rows as a language model gives them: frequent words first, and every history with favourites of its own."""
    z = torch.randn((N, V), generator=g, device=DEVICE)
    z.mul_(2.0).sub_(1.1 * torch.log(torch.arange(1, V + 1, device=DEVICE, dtype=torch.float32)))
    return z.to(DTYPES[dtype])


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    s = dict(case)
    if case["op"] == "q4":
        B, V, H = case["B"], case["V"], case["H"]
        groups, row = -(-H // case["group"]), -(-H // 2)
        # nibbles as a rounded normal weight has them, the even unit in the low half
        n = torch.randn((V, row), generator=g, device=DEVICE)
        codes = n.mul_(3.0).add_(8.0).round_().clamp_(0, 15).to(torch.uint8)
        n.normal_(generator=g)
        codes |= n.mul_(3.0).add_(8.0).round_().clamp_(0, 15).to(torch.uint8) << 4
        del n
        s["codes"] = codes
        s["scales"] = ((torch.rand((groups, V), generator=g, device=DEVICE) + 0.5) * 0.01).to(DTYPES[case["scale"]])
        s["zeros"] = torch.randint(6, 11, (groups, V), generator=g, device=DEVICE, dtype=torch.uint8) if case["zero"] else None
        s["bias"] = torch.randn(V, generator=g, device=DEVICE) * 0.1
        s["rows"] = torch.sigmoid(torch.randn((B, H), generator=g, device=DEVICE)).to(DTYPES[case["x"]])
        s["out"] = torch.empty((B, V), device=DEVICE, dtype=DTYPES[case["y"]])
        return s
    N, V = case["N"], case["V"]
    if case["op"] == "sample":
        z = _logits(g, N, V, case["dtype"])
        s["logits"] = z.masked_fill_(torch.rand((1, V), generator=g, device=DEVICE) < 0.02, -math.inf)  # words that may not come
        r = torch.rand((5, N), generator=g, device=DEVICE)
        kind = {"both": 0, "top_p": 1, "top_k": 2, "min_p": 3, "none": 4, "mixed": -1}[case["rule"]]
        kinds = torch.arange(N, device=DEVICE) % 6 if kind < 0 else torch.full((N,), kind, device=DEVICE)
        s["temperature"] = torch.where(kinds == 5, torch.zeros_like(r[0]), 0.6 + 0.8 * r[0])
        s["top_k"] = torch.where((kinds == 0) | (kinds == 2), torch.exp(math.log(400.0) * r[1]).int() + 1, 0).int()
        s["top_p"] = torch.where(kinds < 2, 0.5 + 0.49 * r[2], 1.0)
        s["min_p"] = torch.where(kinds == 3, 0.01 + 0.19 * r[3], 0.0)
        s["u"] = torch.rand(N, generator=g, device=DEVICE)
        s["word"] = torch.empty(N, dtype=torch.int32, device=DEVICE)
        s["logprob"] = torch.empty(N, device=DEVICE)
        s["workspace"] = None
        return s
    z = _logits(g, N, V, "f32")
    teacher = z + torch.randn((N, V), generator=g, device=DEVICE)
    K = min(case["K"], V)
    s["teacher_logit"], words = teacher.topk(K, dim=1)
    del teacher
    s["teacher_word"] = words.int()
    s["teacher_word"][:, K - K // 8:] = torch.where(torch.rand((N, 1), generator=g, device=DEVICE) < 0.2, -1, s["teacher_word"][:, K - K // 8:])  # shorter lists
    s["logits"] = z.to(DTYPES[case["dtype"]])
    label = torch.randint(0, V, (N,), generator=g, device=DEVICE).int()
    s["labels"] = torch.where(torch.rand(N, generator=g, device=DEVICE) < 0.1, -1, label).int() if case["label"] else None
    s["label_weight"] = 0.25 if case["label"] else 0.0
    s["row_weight"] = torch.rand(N, generator=g, device=DEVICE) / N
    # the statistics that the forward pass keeps for the backward one: the row's maximum, 1 / sum exp((z - max) / T), 1 / sum exp(z - max), 0
    z, T = s["logits"].float(), case["T"]
    top = z.amax(1)
    d = z.sub_(top[:, None])
    s["stats"] = torch.stack([top, 1 / torch.exp(d / T).sum(1), 1 / torch.exp(d).sum(1), torch.zeros_like(top)], 1).contiguous()
    s["loss"] = torch.empty(N, device=DEVICE)
    s["grad"] = torch.empty_like(s["logits"])
    s["workspace"] = None
    return s


# ----------------------------------------------------------------------------------------------------------- plain forms
def _plain_q4(s):
    codes, H, group = s["codes"], s["H"], s["group"]
    w = torch.stack([codes & 15, codes >> 4], dim=2).reshape(s["V"], -1)[:, :H].float()
    of = torch.arange(H, device=DEVICE) // group
    zero = s["zeros"].float() if s["zeros"] is not None else torch.full_like(s["scales"], 8.0, dtype=torch.float32)
    w = (w - zero.t()[:, of]) * s["scales"].float().t()[:, of]
    return (s["rows"].float() @ w.t() + s["bias"]).to(s["out"].dtype)


def _plain_sample(s):
    # in 64 bits: a border between two words is a sum of up to a million others
    z, V = s["logits"].double(), s["V"]
    T = s["temperature"].double()[:, None]
    ordered, order = s["logits"].sort(dim=1, descending=True, stable=True)
    top = z.amax(1, keepdim=True)
    w = torch.exp((ordered.double() - top) / torch.where(T == 0, 1.0, T))
    rank = torch.arange(V, device=DEVICE)
    k = torch.where(s["top_k"] > 0, s["top_k"], V)[:, None]
    w = torch.where(rank < k, w, 0.0)
    before = w.cumsum(1)
    total = before[:, -1:]
    before = before - w
    p = s["top_p"].double()[:, None]
    keep = ((before < p * total) | (p >= 1) | (rank == 0)) & (w >= s["min_p"].double()[:, None])
    w = torch.where(keep, w, 0.0)
    by_word = torch.zeros_like(z).scatter_(1, order, w)
    upto = by_word.cumsum(1)
    total = upto[:, -1:]
    word = (upto <= s["u"].double()[:, None] * total).sum(1, keepdim=True)
    word = torch.where(T == 0, order[:, :1], word.clamp_(max=V - 1))
    logprob = torch.where(T == 0, 0.0, torch.log(by_word.gather(1, word) / total))
    return word[:, 0].int(), logprob[:, 0].float()


def _plain_distill(s):
    z, T, a = s["logits"].float(), s["T"], s["label_weight"]
    there = s["teacher_word"] >= 0
    words = s["teacher_word"].clamp(min=0).long()
    t = torch.where(there, s["teacher_logit"], -math.inf) / T
    t = t - t.amax(1, keepdim=True)
    q = torch.exp(t)
    mass = q.sum(1, keepdim=True)
    q = q / mass
    out = {}
    if s["part"] == "backward":
        top, at_T, at_1 = (s["stats"][:, i:i + 1] for i in range(3))
    else:
        top = z.amax(1, keepdim=True)
        sum_T, sum_1 = torch.exp((z - top) / T).sum(1, keepdim=True), torch.exp(z - top).sum(1, keepdim=True)
        at_T, at_1 = 1 / sum_T, 1 / sum_1
        log_p = (z.gather(1, words) - top) / T - torch.log(sum_T)
        log_q = t - torch.log(mass)
        loss = (1 - a) * T * T * torch.where(there, q * (log_q - log_p), 0.0).sum(1)
        if s["labels"] is not None:
            label = s["labels"].clamp(min=0).long()[:, None]
            loss = loss + a * torch.where(s["labels"] >= 0, (torch.log(sum_1) - (z.gather(1, label) - top))[:, 0], 0.0)
        out["loss"] = loss
        out["stats"] = torch.cat([top, at_T, at_1], 1)
    if s["part"] != "loss":
        g = s["row_weight"][:, None]
        d = (g * (1 - a) * T) * (torch.exp((z - top) / T) * at_T)
        d.scatter_add_(1, words, torch.where(there, -g * (1 - a) * T * q, 0.0))
        if s["labels"] is not None:
            has = (s["labels"] >= 0).float()[:, None]
            d += (g * a * has) * (torch.exp(z - top) * at_1)
            d.scatter_add_(1, s["labels"].clamp(min=0).long()[:, None], -g * a * has)
        out["grad"] = d.to(s["logits"].dtype)
    return out


# ------------------------------------------------------------------------------------------------------- the framework's
def _own_q4(s):
    import paper_2007_11794_amd as rn
    rn.rnnlm_q4_matvec(s["codes"], s["scales"], s["group"], s["rows"], s["out"], zeros=s["zeros"], bias=s["bias"])
    return s["out"]


def _own_sample(s):
    import paper_2007_11794_amd as rn
    if s["workspace"] is None:  # a program makes it once for its sizes
        s["workspace"] = torch.empty(rn.rnnlm_sample_workspace_bytes(s["N"], s["V"]), dtype=torch.uint8, device=DEVICE)
    rn.rnnlm_sample(s["logits"], s["u"], s["word"], s["logprob"], s["workspace"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                    min_p=s["min_p"])
    return s["word"], s["logprob"]


def _own_distill(s):
    import paper_2007_11794_amd as rn
    if s["part"] == "backward":
        rn.rnnlm_distill_backward(s["logits"], s["teacher_word"], s["teacher_logit"], s["stats"], s["grad"], temperature=s["T"], labels=s["labels"],
                                  label_weight=s["label_weight"], row_weight=s["row_weight"])
        return {"grad": s["grad"]}
    if s["workspace"] is None:
        s["workspace"] = torch.empty(rn.rnnlm_distill_workspace_bytes(s["N"], s["V"]), dtype=torch.uint8, device=DEVICE)
    grad = s["grad"] if s["part"] == "step" else None
    rn.rnnlm_distill(s["logits"], s["teacher_word"], s["teacher_logit"], s["loss"], s["stats"], s["workspace"], temperature=s["T"], labels=s["labels"],
                     label_weight=s["label_weight"], row_weight=s["row_weight"], grad=grad)
    out = {"loss": s["loss"], "stats": s["stats"][:, :3]}
    if grad is not None:
        out["grad"] = grad
    return out


def run(state):
    op = state["op"]
    if own:
        return _own_q4(state) if op == "q4" else _own_sample(state) if op == "sample" else _own_distill(state)
    return _plain_q4(state) if op == "q4" else _plain_sample(state) if op == "sample" else _plain_distill(state)


# ------------------------------------------------------------------------------------------------------------------- work
def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["op"] == "q4":
        B, V, H = case["B"], case["V"], case["H"]
        groups = -(-H // case["group"])
        return {"bytes": V * -(-H // 2) + V * groups * (size[case["scale"]] + (1 if case["zero"] else 0)) + V * 4 + B * H * size[case["x"]] + B * V * size[case["y"]],
                "flops": 2 * B * V * H}
    N, V = case["N"], case["V"]
    if case["op"] == "sample":
        return {"bytes": N * V * size[case["dtype"]] + N * 28, "flops": 4 * N * V}
    K, both = min(case["K"], V), 1 if case["part"] == "loss" else 2
    return {"bytes": both * N * V * size[case["dtype"]] + N * K * 8 + N * 28, "flops": both * 4 * N * V}


# --------------------------------------------------------------------------------------------------------- from 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "q4":
        # group by group: what a group's codes add, times its scale
        x, y = s["rows"].double(), s["bias"].double().expand(case["B"], -1).clone()
        for g in range(s["scales"].shape[0]):
            j = torch.arange(g * case["group"], min((g + 1) * case["group"], case["H"]), device=DEVICE)
            c = ((s["codes"][:, j // 2] >> (4 * (j % 2)).to(torch.uint8)) & 15).double()
            off = s["zeros"][g].double() if s["zeros"] is not None else 8.0
            y += s["scales"][g].double() * (x[:, j] @ c.t() - off * x[:, j].sum(1, keepdim=True))
        return y
    if case["op"] == "sample":
        logprob = np.zeros(case["N"])
        rows = s["logits"].double().cpu().numpy()
        T, k, p, m, u = (s[n].double().cpu().numpy() for n in ("temperature", "top_k", "top_p", "min_p", "u"))
        for n in range(case["N"]):
            if T[n] == 0:
                continue
            z = rows[n] / T[n]
            at = np.argsort(-z, kind="stable")
            if k[n] > 0:
                at = at[:int(k[n])]
            e = np.exp(z[at] - z[at[0]])
            if p[n] < 1:
                many = int(np.searchsorted(np.cumsum(e), p[n] * e.sum(), side="left")) + 1
                at, e = at[:many], e[:many]
            at = at[e >= m[n]]
            at.sort()
            e = np.exp(z[at] - z[at].max())
            c = np.cumsum(e)
            logprob[n] = np.log(e[min(int(np.searchsorted(c, u[n] * c[-1], side="right")), len(e) - 1)] / c[-1])
        return [None, logprob]
    z, T, a = s["logits"].double(), case["T"], s["label_weight"]
    N = case["N"]
    if case["part"] == "backward":
        lse_T, lse_1 = (s["stats"][:, :1].double() / c - torch.log(s["stats"][:, i:i + 1].double()) for c, i in ((T, 1), (1.0, 2)))
    else:
        lse_T, lse_1 = torch.logsumexp(z / T, 1, keepdim=True), torch.logsumexp(z, 1, keepdim=True)
    at = [(s["teacher_word"][n] >= 0).nonzero()[:, 0] for n in range(N)]
    loss, sparse = torch.zeros(N, dtype=torch.float64, device=DEVICE), torch.zeros_like(z) if case["part"] != "loss" else None
    for n in range(N):
        w = s["teacher_word"][n, at[n]].long()
        log_q = torch.log_softmax(s["teacher_logit"][n, at[n]].double() / T, 0)
        loss[n] = (1 - a) * T * T * (log_q.exp() * (log_q - z[n, w] / T + lse_T[n])).sum()
        if sparse is not None:
            sparse[n, w] += (1 - a) * T * log_q.exp()
    has = torch.zeros((N, 1), dtype=torch.float64, device=DEVICE)
    if s["labels"] is not None:
        n = (s["labels"] >= 0).nonzero()[:, 0]
        w = s["labels"][n].long()
        has[n] = a
        loss[n] += a * (lse_1[n, 0] - z[n, w])
        if sparse is not None:
            sparse[n, w] += a
    out = {}
    if case["part"] != "backward":
        top = z.amax(1, keepdim=True)
        out["loss"] = loss
        out["stats"] = torch.cat([top, torch.exp(top / T - lse_T), torch.exp(top - lse_1)], 1)
    if sparse is not None:
        d = (1 - a) * T * torch.exp(z / T - lse_T)
        d += has * torch.exp(z - lse_1)
        out["grad"] = (d - sparse) * s["row_weight"].double()[:, None]
    return out
