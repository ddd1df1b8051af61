"""Measured cases of the operators around a serving cache: attention with a causal mask, a sliding window and first tokens
that stay visible, over a plain cache (kvs_window_attention) and over one held in 4 bits (kvs_window_attention_packed), and
the conversions between the two kinds of cache (kvs_pack, kvs_unpack).

A case is a dict of plain values; prepare() makes its inputs, run() makes one pass, in plain torch operations where `own` is
false and with the library's calls where it is true, exact() computes the outputs from the definitions in 64 bits.

A cache in 4 bits: every row of D values is D / 32 blocks of 32, and a block is one power of two (a byte, 127 + its exponent)
and 32 numbers out of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives (a nibble each: sign, then the position in that list; the
lower channel in the lower nibble).
"""

import numpy as np
import torch

own = False

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    attention = dict(dtype="bf16", D=128, G=4, W=1, span=0, sinks=32, counts=False)
    return [
        # one new token per head on a short conversation: latency
        dict(attention, name="window, one token, short", op="window", units=8, shortest=777, longest=777),
        # one new token of eight sequences, sliding window over long caches
        dict(attention, name="window, one token, long", op="window", units=64, shortest=32768, longest=32768, span=8192),
        # a chunk of 512 tokens on merged caches of 2048 slots and itself, with the slots' cardinalities, four sequences
        dict(attention, name="window, chunk on merged", op="window", units=32, shortest=2560, longest=2560, W=512, counts=True),
        # a prompt of 8192 tokens through a layer with a sliding window and sinks
        dict(attention, name="window, prompt, sliding", op="window", units=8, shortest=8192, longest=8192, W=8192, span=2048),
        # the same prompt through a layer that sees all of it: the largest
        dict(attention, name="window, prompt, whole", op="window", units=8, shortest=8192, longest=8192, W=8192),
        # a window of 32 queries of seven heads over fp32 caches of odd lengths, the shortest of less than the window
        dict(attention, name="window, ragged, fp32", op="window", dtype="f32", D=64, G=7, W=32, units=10, shortest=21,
             longest=9001, span=1000, sinks=5),
        # one new token per head on a short conversation held in 4 bits: latency
        dict(attention, name="packed, one token, short", op="packed", units=8, shortest=1000, longest=1000),
        # one new token on the merged caches of all layers, with cardinalities
        dict(attention, name="packed, one token, merged", op="packed", units=256, shortest=4096, longest=4096, counts=True),
        # four drafted tokens of eight heads on long caches
        dict(attention, name="packed, drafts, long", op="packed", units=8, shortest=131072, longest=131072, G=8, W=4),
        # a step's new row of every cache, stored and read back: latency
        dict(name="store, one row", op="store", dtype="bf16", D=128, units=256, shortest=1, longest=1),
        # the merged caches of all layers, stored and read back
        dict(name="store, merged", op="store", dtype="bf16", D=128, units=256, shortest=4096, longest=4096),
        # fp32 caches of unequal lengths
        dict(name="store, ragged, fp32", op="store", dtype="f32", D=64, units=100, shortest=100, longest=9000),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    op = rng.choice(("window", "window", "packed", "packed", "store"))
    case = dict(op=op, dtype=rng.choice(("bf16", "bf16", "f32")), D=rng.choice((64, 128)), units=spread(1, 256))
    if op == "store":
        case["longest"] = min(spread(1, 32768), (1 << 20) // case["units"])
    else:
        case |= dict(G=rng.randint(1, 8), span=rng.choice((0, spread(1, 8192))), sinks=rng.choice((0, spread(1, 64))),
                     counts=rng.random() < 0.4)
        case["longest"] = min(spread(1, 65536), (1 << 20) // case["units"])
        # new tokens of each head: one, a few drafts, or a chunk; at most what the largest prompt costs
        most = (1 << 28) // (case["units"] * case["G"] * case["longest"])
        if op == "packed":
            most = min(most, 8)
        case["W"] = max(1, min(most, rng.choice((1, spread(1, 8), spread(1, 2048)))))
    case["shortest"] = rng.choice((case["longest"], max(1, case["longest"] // rng.randint(2, 9))))
    return case


# ---- inputs
def lengths(case):
    """The units' lengths: the case's own, whatever the seed."""
    rng = np.random.default_rng(case["units"] + case["longest"])
    lens = rng.integers(case["shortest"], case["longest"] + 1, case["units"])
    lens[0], lens[-1] = case["shortest"], case["longest"]
    return lens


def torch_type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def rows_like_a_cache(gen, rows, D, keys):
    """Keys that stay alike over neighbouring tokens, with a few channels that are eight times the others, or Values."""
    x = torch.randn(rows, D, generator=gen, device="cuda")
    if keys:
        near = torch.randn(rows // 16 + 1, D, generator=gen, device="cuda")
        x.mul_(0.5).add_(near.repeat_interleave(16, 0)[:rows], alpha=0.87)
        x[:, torch.randperm(D, generator=gen, device="cuda")[: D // 32]] *= 8
    return x


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    lens = lengths(case)
    first = np.concatenate([[0], np.cumsum(lens)[:-1]])
    rows, D, t = int(lens.sum()), case["D"], torch_type(case)
    s = dict(case=case, lens=lens, first=first, K=rows_like_a_cache(gen, rows, D, True).to(t))
    V = rows_like_a_cache(gen, rows, D, False)
    if case.get("counts"):
        # slots of a merged cache: a Value is the sum over the slot's tokens
        s["counts"] = torch.empty(rows, device="cuda").exponential_(1 / 3, generator=gen).to(torch.int32) + 1
        V *= s["counts"][:, None].sqrt()
    s["V"] = V.to(t)
    if case["op"] != "store":
        s["Q"] = torch.randn(case["units"], case["G"], case["W"], D, generator=gen, device="cuda").to(t)
        s["lens_gpu"], s["first_gpu"] = torch.from_numpy(lens).cuda(), torch.from_numpy(first).cuda()
    if case["op"] == "packed":
        for name in ("K", "V"):
            s[name + "_codes"], s[name + "_scales"] = packed(s.pop(name).float())
    if own:
        s["plan"] = plan(s)
    return s


def plan(s):
    """What a program keeps from call to call: the problem's tables, output buffers, the workspace."""
    import paper_2603_00907_amd as kvs
    case, lens = s["case"], s["lens"]
    attention = case["op"] != "store"
    p = kvs.Problem(lens=lens, budgets=lens, group=case.get("G", 1), window=case.get("W", 1), head_dim=case["D"],
                    dtype=case["dtype"], n_sink=case.get("sinks", 0), causal=attention)
    if attention:
        size = kvs.kvs_window_attention_workspace_size(p, span=case["span"])
        return kvs, p, torch.empty_like(s["Q"]), torch.empty(size, dtype=torch.uint8, device="cuda")
    rows, D = s["K"].shape
    stored = [torch.empty(rows, D // per, dtype=torch.uint8, device="cuda") for per in (2, 32, 2, 32)]
    return kvs, p, stored, [torch.empty_like(s["K"]), torch.empty_like(s["V"])]


# ---- one pass
def run(s):
    case = s["case"]
    if own:
        kvs, p, *buffers = s["plan"]
        stream = torch.cuda.current_stream().cuda_stream
        if case["op"] == "store":
            stored, back = buffers
            kvs.kvs_pack(p, s["K"], s["V"], *stored, stream=stream)
            kvs.kvs_unpack(p, *stored, *back, stream=stream)
            return back
        out, ws = buffers
        if case["op"] == "window":
            kvs.kvs_window_attention(p, s["Q"], s["K"], s["V"], s.get("counts"), out, ws, span=case["span"], stream=stream)
        else:
            kvs.kvs_window_attention_packed(p, s["Q"], s["K_codes"], s["K_scales"], s["V_codes"], s["V_scales"],
                                            s.get("counts"), out, ws, span=case["span"], stream=stream)
        return out
    if case["op"] == "store":
        return [values(*packed(s[name].float())).to(s[name].dtype) for name in ("K", "V")]
    if case["op"] == "packed":
        return attention(s, values(s["K_codes"], s["K_scales"]), values(s["V_codes"], s["V_scales"]))
    return attention(s, s["K"].float(), s["V"].float())


def packed(x):
    """Codes [rows, D / 2] and scales [rows, D / 32] of fp32 rows: a block's scale is the smallest power of two with which none
    of its values rounds beyond 6; values round to the nearest of the grid, from halfway to the one with the even position."""
    rows, D = x.shape
    x = x.view(rows, D // 32, 32)
    part, exponent = torch.frexp(x.abs().amax(-1))  # amax = part 2^exponent, part in [0.5, 1)
    exponent = torch.where(part >= 0.875, exponent - 2, exponent - 3)
    exponent = torch.where(part == 0, -125, exponent).clamp(-125, 125)
    a = torch.ldexp(x.abs(), -exponent[..., None])
    # the halfway points between neighbours of the grid; one that belongs to the upper neighbour counts from itself on
    code = sum((a >= h if up else a > h).to(torch.uint8)
               for h, up in ((0.25, 0), (0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0)))
    code = (code + 8 * (x < 0).to(torch.uint8)).view(rows, D // 2, 2)
    return code[..., 0] + 16 * code[..., 1], (exponent + 127).to(torch.uint8)


def values(codes, scales):
    """The fp32 rows that codes and scales stand for."""
    rows, half = codes.shape
    grid = torch.tensor(GRID + tuple(-g for g in GRID), device=codes.device)
    x = grid[torch.stack([codes & 15, codes >> 4], -1).long()].view(rows, -1, 32)
    return torch.ldexp(x, scales[..., None].to(torch.int32) - 127).view(rows, 2 * half)


def attention(s, K, V):
    """Attention of every unit's G * W query rows over its cache rows that the mask leaves, in fp32."""
    case, Q, lens = s["case"], s["Q"], s["lens_gpu"]
    U, G, W, D = Q.shape
    t = torch.arange(case["longest"], device="cuda")
    at = (s["first_gpu"][:, None] + t).clamp_(max=K.shape[0] - 1)  # [U, n]
    seen = visible(case, lens[:, None] - W + torch.arange(W, device="cuda"), t)  # [U, W, n]
    e = (Q.float().view(U, G * W, D) * D ** -0.5 @ K[at].transpose(1, 2)).view(U, G, W, -1)
    e = e.masked_fill_(~seen[:, None], -torch.inf)
    p = e.sub_(e.amax(-1, keepdim=True).clamp_(min=-1e30)).exp_()
    total = p @ s["counts"][at].float()[:, None, :, None] if case["counts"] else p.sum(-1, keepdim=True)
    out = (p.view(U, G * W, -1) @ V[at]).view(U, G, W, D) / total
    return out.masked_fill_(total == 0, 0.0).to(Q.dtype)


def visible(case, position, t):
    """Which rows t a query at `position` sees: none after it, the last `span` up to it (0: all), the first `sinks`."""
    position = position[..., None]
    near = t > position - case["span"] if case["span"] else t >= 0
    return (t <= position) & (near | (t < case["sinks"]))


# ---- what a pass cannot do without
def work(case):
    size, D = (4 if case["dtype"] == "f32" else 2), case["D"]
    lens = lengths(case)
    if case["op"] == "store":
        return {"bytes": int(2 * lens.sum() * (2 * D * size + 2 * (D // 2 + D // 32))), "flops": 0}
    row = 2 * (D * size if case["op"] == "window" else D // 2 + D // 32) + (4 if case["counts"] else 0)
    pairs = rows = 0
    for n in lens:
        last = np.arange(max(0, n - case["W"]), n)  # the queries' positions
        span, sinks = (case["span"] or int(n)), case["sinks"]
        pairs += int(np.minimum(last + 1, span + np.clip(last + 1 - span, 0, sinks)).sum())
        first = max(0, int(last[0]) - span + 1)
        rows += int(n) - first + min(sinks, first)
    return {"bytes": rows * row + 2 * case["units"] * case["G"] * case["W"] * D * size, "flops": 4 * D * case["G"] * pairs}


# ---- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "store":
        return [nearest(s["K"].double()), nearest(s["V"].double())]
    if case["op"] == "packed":
        K, V = (stands_for(s[x + "_codes"], s[x + "_scales"]) for x in "KV")
    else:
        K, V = s["K"].double(), s["V"].double()
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    W = case["W"]
    for u, (n, r) in enumerate(zip(s["lens"].tolist(), s["first"].tolist())):
        keys, vals = K[r:r + n], V[r:r + n]
        c = s["counts"][r:r + n].double() if case["counts"] else torch.ones(n, dtype=torch.float64, device="cuda")
        behind = torch.arange(n - W, n, device="cuda")[:, None] - torch.arange(n, device="cuda")  # how far behind the query
        hidden = behind < 0
        if case["span"]:
            hidden |= (behind >= case["span"]) & (torch.arange(n, device="cuda") >= case["sinks"])
        some = ~hidden.all(1)
        for g in range(case["G"]):
            e = s["Q"][u, g].double() @ keys.T / np.sqrt(case["D"])
            e[hidden] = -torch.inf
            e = torch.exp(e - torch.logsumexp(e + c.log(), 1, keepdim=True))
            out[u, g, some] = (e @ vals)[some]
    return out


def nearest(x):
    """What a row of 64-bit numbers stands for after it was held in 4 bits."""
    rows, D = x.shape
    x = x.view(-1, 32)
    a = x.abs()
    top = a.amax(1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -140))).clamp(-130, 130)
    e = e + (2.0 ** (e + 1) <= top).double() - (2.0 ** e > top).double()  # 2^e <= top < 2^(e+1), whatever log2 rounds to
    e = (e - 2 + (top >= 1.75 * 2.0 ** e).double()).clamp(-125, 125)
    a = a / 2.0 ** e
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    return (torch.round(a / step) * step).clamp(max=6).copysign(x).mul(2.0 ** e).view(rows, D)


def stands_for(codes, scales):
    nibbles = torch.stack([codes % 16, codes // 16], -1).flatten(1).long()
    e, m = nibbles % 8 // 2, (nibbles % 2).double()
    size = torch.where(e == 0, m / 2, (1 + m / 2) * 2.0 ** (e - 1).double())
    return torch.where(nibbles >= 8, -size, size) * (2.0 ** (scales.double() - 127)).repeat_interleave(32, 1)
