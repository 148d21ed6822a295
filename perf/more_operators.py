"""The gated feed-forward block on quantized weights, and the loss of the vocabulary projection with its gradient.

The linears of a decoder layer are quantized; between and behind them a training step and a generation step need two
more operators.  A case names one kind of work (``op``) and its sizes:

  glu_fwd     H = act(X Wg^T) * (X Wu^T), gate and up projection quantized; with ``keep`` the two products, Y, are kept for
              the backward pass
  glu_bwd     from dH and Y the gradient dY of both products, which the backward pass of the linear that they are goes on from
  glu_decode  H of 1 to 16 new tokens from the prepared weights; ``tasks`` > 0: every token with the scales of its own task
  loss        softmax cross entropy of the logits X W^T of a vocabulary of ``vocab`` tokens, each token's loss, and with
              ``grad`` the gradient of their weighted sum with respect to X (W is frozen).  Tokens with a negative label
              count nothing; ``masked``: all but the answers of instruction samples are such tokens.

Gate and up projection are one quantized linear of 2 * ``ffn`` rows, in which runs of eight rows of the gate alternate with the
eight rows of the up projection for the same channels.  ``width`` is the layer's width; ``bits`` and ``group`` (0: one scale
per row) as everywhere.
"""
import math

import torch

own = False


def _glu(name, op, tokens, ffn, width, bits, group, act="silu", keep=False, tasks=0):
    named = {} if name is None else {"name": name}
    return named | {"op": op, "tokens": tokens, "ffn": ffn, "width": width, "bits": bits, "group": group, "act": act,
                    "keep": keep, "tasks": tasks}


def _back(name, tokens, ffn, act="silu"):
    named = {} if name is None else {"name": name}
    return named | {"op": "glu_bwd", "tokens": tokens, "ffn": ffn, "act": act}


def _loss(name, tokens, vocab, width, grad, masked=False):
    named = {} if name is None else {"name": name}
    return named | {"op": "loss", "tokens": tokens, "vocab": vocab, "width": width, "grad": grad, "masked": masked}


def listed():
    return [
        # generation, LLaMA-7B MLP, one sequence: the latency of a chat server
        _glu("glu_decode_1", "glu_decode", 1, 11008, 4096, 4, 0),
        # a full serving batch on LLaMA-65B's MLP, groups of 64
        _glu("glu_decode_16", "glu_decode", 16, 22016, 8192, 3, 64),
        # several users, each with the scales of their own task
        _glu("glu_decode_tasks_7", "glu_decode", 7, 11008, 4096, 3, 128, tasks=4),
        # a short prompt
        _glu("glu_prompt_77", "glu_fwd", 77, 11008, 4096, 4, 128),
        # forward of a training step, LLaMA-7B's MLP, one scale per channel (the paper's main setting), two 2048-token sequences
        _glu("glu_train_7b", "glu_fwd", 4096, 11008, 4096, 4, 0, keep=True),
        # backward of a ragged batch of short instruction samples, a block with the other activation
        _back("glu_back_ragged", 1001, 11008, act="gelu_tanh"),
        # backward of LLaMA-65B's MLP, 4096 tokens
        _back("glu_back_65b", 4096, 22016),
        # one token's log-probability: the smallest
        _loss("loss_1_token", 1, 32000, 4096, False),
        # perplexity of one 2048-token sequence
        _loss("loss_eval_7b", 2048, 32000, 4096, False),
        # a short sample alone
        _loss("loss_train_short", 150, 32000, 4096, True),
        # the end of a training step of LLaMA-65B, 4096 tokens: the largest
        _loss("loss_train_65b", 4096, 32000, 8192, True),
        # instruction tuning on a larger vocabulary of an odd size: loss on the answers alone
        _loss("loss_train_masked", 4091, 50257, 4096, True, masked=True),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


#: products (tokens * rows * width) that no drawn case goes beyond
_MOST_GLU = 4096 * 22016 * 8192
_MOST_LOSS = 4096 * 32000 * 8192


def draw(rng):
    op = rng.choice(["glu_decode", "glu_fwd", "glu_bwd", "loss", "loss"])
    if op == "loss":
        vocab, width = _log_uniform(rng, 1000, 131072), 8 * _log_uniform(rng, 32, 1024)
        grad = rng.random() < 0.6
        tokens = _log_uniform(rng, 1, min(8192, _MOST_LOSS // (vocab * width), (1 << 28) // vocab))
        return _loss(None, tokens, vocab, width, grad, tokens >= 400 and rng.random() < 0.4)
    bits, act = rng.choice([3, 4]), rng.choice(["silu", "silu", "gelu_tanh"])
    ffn, width = 8 * _log_uniform(rng, 16, 2752), 128 * _log_uniform(rng, 2, 64)
    if op == "glu_bwd":
        return _back(None, _log_uniform(rng, 1, 8192), ffn, act)
    group = rng.choice([0, 0] + [g for g in (64, 128, 256) if width % g == 0])
    if op == "glu_decode":
        return _glu(None, op, rng.randrange(1, 17), ffn, width, bits, group, act, tasks=rng.choice([0, 0, 3]))
    tokens = _log_uniform(rng, 17, min(8192, _MOST_GLU // (ffn * width)))
    return _glu(None, op, tokens, ffn, width, bits, group, act, keep=op == "glu_fwd" and rng.random() < 0.5)


def _groups(case):
    return 1 if case["group"] in (0, case["width"]) else case["width"] // case["group"]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
    T = case["tokens"]
    s = {"case": case}
    if case["op"] == "glu_bwd":
        s["Y"], s["dH"] = 1.5 * randn(T, 2 * case["ffn"]), randn(T, case["ffn"]) * 2.0 ** -6
        return s
    K = case["width"]
    if case["op"] == "loss":
        V = case["vocab"]
        s["W"] = (randn(V, K) * K ** -0.5)                        # logits of unit size from a normalised hidden state
        labels = torch.randint(V, (T,), generator=gen, device="cuda")
        # some tokens are foregone conclusions, others mere guesses: up to 14 of logit towards the label
        sure = torch.rand((T, 1), generator=gen, device="cuda") * 14
        s["X"] = (randn(T, K).float() + sure * s["W"][labels].float()).bfloat16()
        if case["masked"]:                                        # samples of 200 tokens, the last 80 an answer
            labels = torch.where(torch.arange(T, device="cuda") % 200 < 120, -100, labels)
        s["labels"] = labels.int()
        # the mean over the tokens that count, and 8 as the scale of a step in 16 bits
        s["weight"] = torch.full((T,), 8.0 / max(1, int((labels >= 0).sum())), device="cuda")
        return s
    N, G, bits = 2 * case["ffn"], _groups(case), case["bits"]
    # any bits are codes; scales about as large as a weight matrix of unit gain has them
    s["words"] = torch.randint(-2 ** 31, 2 ** 31, (N, K * bits // 32), generator=gen, device="cuda").int()
    s["zeros"] = torch.randint(2 ** (bits - 1) - 1, 2 ** (bits - 1) + 1, (N, G), generator=gen, device="cuda").to(torch.uint8)
    size = (case["tasks"],) if case["tasks"] else ()
    s["scales"] = (0.5 + torch.rand(size + (N, G), generator=gen, device="cuda")) * (K ** -0.5 * 3.5 / 2 ** bits)
    s["X"] = randn(T, K)
    if case["tasks"]:
        s["ids"] = torch.randint(case["tasks"], (T,), generator=gen, device="cuda").int()
    return s


def _handle(s):
    """The framework's descriptor of the block and what it works in: made once, as a program would."""
    if "binding" not in s:
        from paper_2305_14152_b200 import binding
        case = s["case"]
        s["binding"] = binding
        if case["op"] == "loss":
            s["workspace"] = binding.alloc_head_loss_workspace(s["X"], s["W"], case["grad"])
        elif case["op"] != "glu_bwd":
            s["w"] = binding.QWeight(case["bits"], 2 * case["ffn"], case["width"], case["group"], s["words"], s["zeros"],
                                     s["scales"][0] if case["tasks"] else s["scales"])
            if case["op"] == "glu_decode":
                s["prepared"] = binding.decode_prepare(s["w"])
    return s["binding"]


# ---------------------------------------------------------------------------------------------- plain forms

def _codes(words, bits):
    """Codes of packed rows, [rows, columns]: column j is bits [bits * j, bits * j + bits) of a row's little-endian bit string."""
    if bits == 4:
        return ((words[:, :, None] >> (4 * torch.arange(8, device="cuda", dtype=torch.int32))) & 15).flatten(1)
    w = (words.long() & 0xFFFFFFFF).view(words.shape[0], -1, 3)
    low, high = w[:, :, 0] | w[:, :, 1] << 32, w[:, :, 1] | w[:, :, 2] << 32
    shift = 3 * torch.arange(32, device="cuda")
    return torch.cat([low[:, :, None] >> shift[:21], high[:, :, None] >> shift[21:] - 32], 2).flatten(1) & 7


def _weights(s, scales, dtype):
    """s * (Q - z), a few thousand rows at a time, as their codes take eight bytes each on the way."""
    N, K = s["words"].shape[0], s["case"]["width"]
    out = torch.empty((N, K), dtype=dtype, device="cuda")
    for i in range(0, N, 4096):
        rows = slice(i, i + 4096)
        q = _codes(s["words"][rows], s["case"]["bits"]).to(dtype).view(-1, scales.shape[1], K // scales.shape[1])
        out[rows] = ((q - s["zeros"][rows, :, None].to(dtype)) * scales[rows, :, None].to(dtype)).flatten(1)
    return out


def _gates(x, act):
    """Both activations are x * p(v), p the logistic function, with v = x, or 2 sqrt(2/pi) (x + 0.044715 x^3): p, 1 - p and dv/dx."""
    c = 2 * math.sqrt(2 / math.pi)
    v, slope = (x, torch.ones_like(x)) if act == "silu" else (c * (x + 0.044715 * x ** 3), c * (1 + 3 * 0.044715 * x * x))
    return 1 / (1 + torch.exp(-v)), 1 / (1 + torch.exp(v)), slope


def _act(x, act):
    return x * _gates(x, act)[0]


def _act_slope(x, act):
    p, q, slope = _gates(x, act)
    return p * (1 + x * q * slope)


def _halves(y):
    """Gate and up side of [tokens, 2 * ffn]: runs of eight by turns."""
    y = y.view(y.shape[0], -1, 2, 8)
    return y[:, :, 0].flatten(1), y[:, :, 1].flatten(1)


def _glu_forward(s):
    case = s["case"]
    X = s["X"].float()
    if case["tasks"]:
        Y = torch.empty((case["tokens"], 2 * case["ffn"]), device="cuda")
        for task in range(case["tasks"]):
            mine = (s["ids"] == task)[:, None]
            Y = torch.where(mine, X @ _weights(s, s["scales"][task], torch.float32).T, Y)
    else:
        Y = X @ _weights(s, s["scales"], torch.float32).T
    gate, up = _halves(Y)
    H = (_act(gate, case["act"]) * up).bfloat16()
    return (H, Y.bfloat16()) if case["keep"] else H


def _glu_backward(s):
    act, dH = s["case"]["act"], s["dH"].float()
    gate, up = _halves(s["Y"].float())
    d = [(dH * up * _act_slope(gate, act)).unflatten(1, (-1, 8)), (dH * _act(gate, act)).unflatten(1, (-1, 8))]
    return torch.stack(d, 2).flatten(1).bfloat16()


def _loss_plain(s):
    counts = s["labels"] >= 0
    X, W, labels = s["X"][counts].float(), s["W"].float(), s["labels"][counts].long()[:, None]
    logits = X @ W.T
    of_label = logits.gather(1, labels)
    most = logits.amax(1, keepdim=True)
    p = torch.exp(logits - most)
    total = p.sum(1, keepdim=True, dtype=torch.float64)            # in 64 bits: the loss of a sure token is next to nothing
    loss = torch.zeros(s["labels"].shape, device="cuda")
    loss[counts] = (torch.log(total) + most - of_label)[:, 0].float()
    if not s["case"]["grad"]:
        return loss
    p /= total.float()
    p.scatter_add_(1, labels, torch.full_like(of_label, -1.0))
    dX = torch.zeros_like(s["X"])
    dX[counts] = ((p @ W) * s["weight"][counts][:, None]).bfloat16()
    return loss, dX


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return _loss_plain(s) if op == "loss" else _glu_backward(s) if op == "glu_bwd" else _glu_forward(s)
    binding = _handle(s)
    if op == "loss":
        loss, dX = binding.head_loss(s["X"], s["W"], s["labels"], s["weight"], need_grad=case["grad"], workspace=s["workspace"])
        return (loss, dX) if case["grad"] else loss
    if op == "glu_bwd":
        return binding.glu_bwd(s["Y"], s["dH"], case["act"])
    if op == "glu_fwd":
        H, Y = binding.qglu_fwd(s["w"], s["X"], case["act"], keep=case["keep"])
        return (H, Y) if case["keep"] else H
    table, ids = (s["scales"], s["ids"]) if case["tasks"] else (None, None)
    return binding.qglu_decode_prepared(s["w"], s["prepared"], s["X"], case["act"], scale_table=table, task_ids=ids)


def work(case):
    T = case["tokens"]
    if case["op"] == "glu_bwd":
        return {"bytes": 2 * T * 5 * case["ffn"], "flops": 20 * T * case["ffn"]}
    K = case["width"]
    if case["op"] == "loss":
        V = case["vocab"]
        live = sum(1 for t in range(T) if t % 200 >= 120) if case["masked"] else T
        rows = live * 2 * K + 8 * T + (2 * T * K + 4 * T if case["grad"] else 0)
        return {"bytes": 2 * V * K + rows, "flops": (4 if case["grad"] else 2) * live * V * K}
    N, G = 2 * case["ffn"], _groups(case)
    weights = N * K * case["bits"] // 8 + N * G
    scales = 4 * N * G * (min(T, case["tasks"]) if case["tasks"] else 1)
    return {"bytes": weights + scales + 2 * T * (K + N // 2 + (N if case["keep"] else 0)), "flops": 2 * T * N * K}


def exact(case, seed):
    s = prepare(case, seed)
    T = case["tokens"]
    if case["op"] == "glu_bwd":
        gate, up, dH = (t.double() for t in (*_halves(s["Y"]), s["dH"]))
        if case["act"] == "silu":
            a = gate * torch.sigmoid(gate)
            slope = torch.sigmoid(gate) + a * torch.sigmoid(-gate)
        else:
            c, k = math.sqrt(2 / math.pi), 0.044715
            inner = c * (gate + k * gate ** 3)
            a = 0.5 * gate * (1 + torch.tanh(inner))
            slope = 0.5 * (1 + torch.tanh(inner)) + 0.5 * gate / torch.cosh(inner) ** 2 * c * (1 + 3 * k * gate ** 2)
        return torch.cat([(dH * up * slope).view(T, -1, 1, 8), (dH * a).view(T, -1, 1, 8)], 2).view(T, -1)
    X = s["X"].double()
    if case["op"] == "loss":
        W = s["W"].double()
        loss = torch.zeros(T, dtype=torch.float64, device="cuda")
        dX = torch.zeros(X.shape, dtype=torch.float64, device="cuda")
        rows = (s["labels"] >= 0).nonzero()[:, 0]
        for part in rows.split(512):                              # logits of a few tokens at a time
            logits = X[part] @ W.T
            label = s["labels"][part].long()
            rest = logits - logits[torch.arange(len(part), device="cuda"), label][:, None]
            total = torch.logsumexp(rest, 1)
            loss[part] = total
            if case["grad"]:
                p = torch.exp(rest - total[:, None])
                dX[part] = (p @ W - W[label]) * s["weight"][part].double()[:, None]
        return (loss, dX) if case["grad"] else loss
    tables = s["scales"] if case["tasks"] else s["scales"][None]
    ids = s["ids"].tolist() if case["tasks"] else [0] * T
    Y = torch.empty((T, 2 * case["ffn"]), dtype=torch.float64, device="cuda")
    for task in sorted(set(ids)):
        mine = torch.tensor([i for i, t in enumerate(ids) if t == task], device="cuda")
        Y[mine] = X[mine] @ _weights(s, tables[task], torch.float64).T
    gate, up = _halves(Y)
    if case["act"] == "silu":
        H = gate * torch.sigmoid(gate) * up
    else:
        H = 0.5 * gate * (1 + torch.tanh(math.sqrt(2 / math.pi) * (gate + 0.044715 * gate ** 3))) * up
    return (H, Y) if case["keep"] else H
