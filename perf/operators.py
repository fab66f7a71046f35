"""The 8-bit operators as cases that can be timed and compared with their plain forms.

A case is a dict of plain values; `op` says which operator:
  quant_i8   rows of a matrix to 8-bit integers with a scale each: tokens online (bf16), weight channels offline (FP32)
  gemm_i8    y = bf16(sx[m] sw[n] sum_k xq[m, k] wq[n, k]) of such operands
  append     new keys and values into a paged cache of 8-bit integers, a scale for each page (block of tokens) and head
  attn       attention of the newest tokens over that cache, causal, grouped query heads
Values: activations N(0, 1) in bf16 with 1 % of the channels twenty times larger; weights Student-t-like; cached keys and values
near N(0, 1).  Sequence lengths of a ragged batch follow from the case alone, page orders and values from the seed.
"""
import math
import random

import torch

own = False


def listed():
    return [
        # One decoded token before an 8-bit projection: next to no work, all latency.
        {"name": "quant_token", "op": "quant_i8", "M": 1, "K": 4096, "fp32": False},
        # A short prompt of odd length into the down projection.
        {"name": "quant_prompt", "op": "quant_i8", "M": 333, "K": 11008, "fp32": False},
        # An MLP weight, quantized once per output channel.
        {"name": "quant_weight", "op": "quant_i8", "M": 11008, "K": 4096, "fp32": True},
        # Decode of one sequence: every weight byte is read for one token.
        {"name": "i8_decode", "op": "gemm_i8", "M": 1, "N": 11008, "K": 4096},
        # A decode batch against the largest projection of a 70B-like model.
        {"name": "i8_batch", "op": "gemm_i8", "M": 16, "N": 28672, "K": 8192},
        # A short prompt that fills no token tile.
        {"name": "i8_ragged", "op": "gemm_i8", "M": 333, "N": 4096, "K": 11008},
        # Prefill of a full prompt.
        {"name": "i8_prefill", "op": "gemm_i8", "M": 2048, "N": 14336, "K": 4096},
        # One decode step of a batch writes one token to each sequence.
        {"name": "append_decode", "op": "append", "B": 64, "n": 1, "ragged": False, "len": 1024, "H": 8, "D": 128, "page": 16},
        # Prompts of different lengths are written whole.
        {"name": "append_prompt", "op": "append", "B": 7, "n": 2048, "ragged": True, "len": 2048, "H": 8, "D": 128, "page": 64},
        # Decode of one sequence of moderate length: latency, and work for all SMs out of a single row of queries.
        {"name": "attn_one", "op": "attn", "B": 1, "n": 1, "ragged": False, "len": 4096, "H": 8, "G": 4, "D": 64, "page": 16},
        # A full decode batch of very different lengths.
        {"name": "attn_batch", "op": "attn", "B": 64, "n": 1, "ragged": True, "len": 16384, "H": 8, "G": 8, "D": 128, "page": 64},
        # Chunks of long prompts, each over what is cached before it.
        {"name": "attn_chunk", "op": "attn", "B": 3, "n": 1000, "ragged": True, "len": 8192, "H": 8, "G": 4, "D": 128, "page": 128},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithms; K is a multiple of 16 (the library's rule), M and N are
    anything."""
    op = rng.choice(["quant_i8", "gemm_i8", "gemm_i8", "append", "attn", "attn", "attn"])
    if op == "quant_i8":
        while True:
            m, k = _log_int(rng, 1, 11008), _log_int(rng, 16, 28672) // 16 * 16
            if m * k <= 11008 * 4096:
                return {"op": op, "M": m, "K": k, "fp32": rng.random() < 0.4}
    if op == "gemm_i8":
        while True:
            m, n, k = _log_int(rng, 1, 2048), _log_int(rng, 64, 28672), _log_int(rng, 64, 28672) // 16 * 16
            if n * k <= 28672 * 8192 and m * n * k <= 2048 * 14336 * 4096:
                return {"op": op, "M": m, "N": n, "K": k}
    while True:
        c = {"op": op, "B": _log_int(rng, 1, 96), "n": 1, "ragged": rng.random() < 0.7, "len": _log_int(rng, 1, 32768), "H": rng.choice([1, 2, 4, 8, 16]),
             "D": rng.choice([64, 128, 128]), "page": rng.choice([16, 32, 64, 128])}
        if rng.random() < 0.5:
            c["n"] = min(c["len"], rng.choice([_log_int(rng, 2, 8), _log_int(rng, 2, 2048)]))
        if op == "append":
            if c["B"] * c["len"] * c["H"] * c["D"] <= 1 << 27:
                return c
            continue
        c["G"] = rng.choice([1, 2, 4, 5, 8, 16])
        padded = c["B"] * -(-c["len"] // c["page"]) * c["page"] * c["H"]
        if padded * c["D"] <= 1 << 29 and padded * c["G"] * c["n"] <= 1 << 29 and work(c)["flops"] < 2e11:
            return c


def _lens(case):
    """([new tokens], [tokens in the cache with the new ones]) of each sequence; ragged ones between an eighth and all of the case's."""
    B, n, length = case["B"], case["n"], case["len"]
    if not case["ragged"]:
        return [n] * B, [length] * B
    rng = random.Random(B * 1000003 + n * 101 + length)
    new = [max(1, int(n * rng.uniform(0.125, 1.0))) if n > 8 else rng.randint(1, n) for _ in range(B)]
    total = [max(1, int(length * rng.uniform(0.125, 1.0))) for _ in range(B)]
    new[0], total[0] = n, length
    return [min(a, b) for a, b in zip(new, total)], total


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    op = case["op"]
    if op == "quant_i8":
        x = randn(case["M"], case["K"])
        if case["fp32"]:
            return {"op": op, "x": 0.02 * x / (randn(case["M"], 1).abs() + 0.5)}
        x[:, torch.randperm(case["K"], generator=g, device="cuda")[: case["K"] // 100 + 1]] *= 20
        return {"op": op, "x": x.bfloat16()}
    if op == "gemm_i8":
        m, n, k = case["M"], case["N"], case["K"]
        codes = lambda r: (32 * randn(r, k)).round_().clamp_(-127, 127).to(torch.int8)  # noqa: E731
        return {"op": op, "x": codes(m), "w": codes(n), "sx": randn(m).abs() * 0.02 + 0.01, "sw": randn(n).abs() * 2e-4 + 2e-4}
    new, total = _lens(case)
    B, H, D, page = case["B"], case["H"], case["D"], case["page"]
    held = [-(-t // page) for t in total]
    pages, width = sum(held) + 3, max(held)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    at = torch.tensor([sum(held[:b]) for b in range(B)], device="cuda")[:, None] + torch.arange(width, device="cuda")
    table = order[at.clamp(max=pages - 1)]
    starts = [sum(new[:b]) for b in range(B + 1)]
    T = starts[-1]
    pool = lambda: (32 * randn(pages, H, page, D)).round_().clamp_(-127, 127).to(torch.int8)  # noqa: E731
    scales = lambda: 0.02 + 0.02 * torch.rand((pages, H), generator=g, device="cuda")  # noqa: E731
    s = {"op": op, "k": pool(), "v": pool(), "ks": scales(), "vs": scales(), "table": table.contiguous(), "T": T, "n_max": max(new), "page": page,
         "q_start": torch.tensor(starts, dtype=torch.int32, device="cuda"), "kv_len": torch.tensor(total, dtype=torch.int32, device="cuda")}
    if op == "append":
        # keys and values as they come out of one projection: columns of a wider matrix
        both = randn(T, 2 * H * D)
        both[:, torch.randperm(2 * H * D, generator=g, device="cuda")[: H * D // 50 + 1]] *= 4
        both = both.bfloat16()
        s["k_new"], s["v_new"] = both[:, : H * D].view(T, H, D), both[:, H * D:].view(T, H, D)
    else:
        s["q"] = randn(T, H * case["G"], D).bfloat16()
    if own:
        from paper_2501_04052_b200 import binding as b
        s["cache"] = b.make_kv8(s["k"], s["v"], s["ks"], s["vs"])
        if op == "attn":
            s["workspace"] = b.alloc_attn_workspace(s["cache"], H * case["G"], "cuda")
    return s


def _tokens(s):
    """(sequence, position) of every new token."""
    t = torch.arange(s["T"], device="cuda")
    seq = torch.searchsorted(s["q_start"][1:].long(), t, right=True)
    return seq, s["kv_len"].long()[seq] - s["q_start"].long()[seq + 1] + t


def _quotients(x, scale):
    """rint(x / scale) with the quotient in 64 bits, so that a value next to a border goes to its own side; 0 where the scale is 0."""
    return (x.double() / torch.where(scale == 0, 1.0, scale).double()).round_().clamp_(-127, 127)


def _plain_append(s):
    seq, pos = _tokens(s)
    page = s["page"]
    col = pos // page
    home = s["table"].long()[seq, col]                                  # the page of every new token
    begun = (s["kv_len"].long() - s["q_start"].long().diff())[seq] < col * page + 1     # no older token in that page
    for codes, scales, x in ((s["k"], s["ks"], s["k_new"]), (s["v"], s["vs"], s["v_new"])):
        high = torch.zeros_like(scales).index_reduce_(0, home, x.float().abs().amax(2), "amax")
        old = scales.index_fill(0, home[begun], 0.0)
        grown = torch.maximum(old, (high.double() / 127).float())
        touched = torch.zeros(scales.shape[0], dtype=torch.bool, device="cuda").index_fill_(0, home, True)
        pages = touched.nonzero()[:, 0]
        was, now = old[pages][..., None, None], grown[pages][..., None, None]
        held = codes[pages]
        codes[pages] = torch.where((was > 0) & (now > was), _quotients(held.double() * was.double(), now).to(torch.int8), held)
        scales.copy_(torch.where(touched[:, None], grown, scales))
        codes[home, :, pos % page] = _quotients(x, scales[home][..., None]).to(torch.int8)
    return s["k"], s["v"], s["ks"], s["vs"]


def _plain_attn(s):
    q, table, page, n_max = s["q"], s["table"].long(), s["page"], s["n_max"]
    B, width = table.shape
    H, D = s["k"].shape[1], q.shape[2]
    G = q.shape[1] // H
    k, v = ((c[table].float() * sc[table][..., None, None]).transpose(1, 2).reshape(B, H, width * page, D) for c, sc in ((s["k"], s["ks"]), (s["v"], s["vs"])))
    seq, pos = _tokens(s)
    row = torch.arange(s["T"], device="cuda") - s["q_start"].long()[seq]
    padded = torch.zeros((B, n_max, H, G, D), device="cuda")
    padded[seq, row] = q.float().view(-1, H, G, D)
    limit = torch.full((B, n_max), -1, device="cuda").index_put_((seq, row), pos)
    scores = (padded.permute(0, 2, 1, 3, 4).reshape(B, H, n_max * G, D) @ k.transpose(2, 3)).mul_(D ** -0.5).view(B, H, n_max, G, width * page)
    hidden = torch.arange(width * page, device="cuda") > limit[:, None, :, None, None]
    scores.masked_fill_(hidden, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_(min=-3e38)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p.view(B, H, n_max * G, -1) @ v).view(B, H, n_max, G, D) / total.clamp(min=1e-38)
    lse = (total.log() + top)[..., 0]
    return out.permute(0, 2, 1, 3, 4)[seq, row].reshape(-1, H * G, D).to(q.dtype), lse.permute(0, 2, 1, 3)[seq, row].reshape(-1, H * G)


def run(s):
    op = s["op"]
    if own:
        from paper_2501_04052_b200 import binding as b
        if op == "quant_i8":
            return b.razer_quant_i8(s["x"])
        if op == "gemm_i8":
            return b.razer_gemm_i8(s["x"], s["sx"], s["w"], s["sw"])
        if op == "append":
            b.razer_kv8_append(s["cache"], s["k_new"], s["v_new"], s["table"], s["q_start"], s["kv_len"])
            return s["k"], s["v"], s["ks"], s["vs"]
        return b.razer_attn_kv8(s["cache"], s["q"], s["table"], s["q_start"], s["kv_len"], workspace=s["workspace"])
    if op == "quant_i8":
        scale = (s["x"].abs().amax(1).double() / 127).float()
        return _quotients(s["x"], scale[:, None]).to(torch.int8), scale
    if op == "gemm_i8":
        return ((s["x"].float() @ s["w"].float().t()) * (s["sx"][:, None] * s["sw"])).bfloat16()
    return _plain_append(s) if op == "append" else _plain_attn(s)


def work(case):
    op = case["op"]
    if op == "quant_i8":
        n = case["M"] * case["K"]
        return {"bytes": n * (5 if case["fp32"] else 3) + 4 * case["M"], "flops": 3 * n}
    if op == "gemm_i8":
        m, n, k = case["M"], case["N"], case["K"]
        return {"bytes": (m + n) * (k + 4) + 2 * m * n, "flops": 2 * m * n * k}
    new, total = _lens(case)
    H, D, page = case["H"], case["D"], case["page"]
    if op == "append":
        touched = sum((t - 1) // page - (t - n) // page + 1 for n, t in zip(new, total))
        return {"bytes": sum(new) * H * D * 6 + 16 * H * touched + 4 * touched, "flops": 6 * sum(new) * H * D}
    rows = sum(new) * H * case["G"]
    pairs = sum(n * t - n * (n - 1) // 2 for n, t in zip(new, total)) * H * case["G"]
    held = sum(-(-t // page) for t in total)
    return {"bytes": 2 * sum(total) * H * D + held * (8 * H + 4) + rows * (4 * D + 4), "flops": 4 * D * pairs}


def exact(case, seed):
    """The operators as they are defined, in 64 bits; sequence by sequence, page by page."""
    s = prepare(case, seed)
    op = case["op"]
    if op == "quant_i8":
        x = s["x"].to(torch.float64)
        step = (x.abs().max(dim=1).values / 127.0).to(torch.float32)
        safe = step.to(torch.float64).masked_fill(step == 0, 1.0)
        return torch.clamp(torch.round(x / safe.unsqueeze(1)), -127, 127).to(torch.int8), step
    if op == "gemm_i8":
        sums = torch.matmul(s["x"].to(torch.float64), s["w"].to(torch.float64).T)
        return sums * s["sx"].to(torch.float64).unsqueeze(1) * s["sw"].to(torch.float64).unsqueeze(0)
    starts, lens, table = s["q_start"].tolist(), s["kv_len"].tolist(), s["table"].tolist()
    page, D = case["page"], case["D"]
    if op == "append":
        for codes, scales, x in ((s["k"], s["ks"], s["k_new"].double()), (s["v"], s["vs"], s["v_new"].double())):
            for b, length in enumerate(lens):
                first = length - (starts[b + 1] - starts[b])
                for c in range(first // page, (length - 1) // page + 1):
                    lo, hi, at = max(first, c * page), min(length, (c + 1) * page), table[b][c]
                    new = x[starts[b] + lo - first:starts[b] + hi - first].transpose(0, 1)
                    step = (new.abs().amax(dim=(1, 2)) / 127.0).float()
                    if lo > c * page:
                        before = scales[at].clone()
                        step = torch.maximum(step, before)
                        ratio = codes[at].double() * before.double()[:, None, None] / step.double().masked_fill(step == 0, 1.0)[:, None, None]
                        codes[at] = torch.where((step > before)[:, None, None] & (before > 0)[:, None, None], torch.round(ratio), codes[at].double()).to(torch.int8)
                    scales[at] = step
                    quotient = new / step.double().masked_fill(step == 0, 1.0)[:, None, None]
                    codes[at, :, lo - c * page:hi - c * page] = torch.clamp(torch.round(quotient), -127, 127).to(torch.int8)
        return s["k"], s["v"], s["ks"], s["vs"]
    H, G = case["H"], case["G"]
    outs, sums = [], []
    for b, length in enumerate(lens):
        n, at = starts[b + 1] - starts[b], torch.tensor(table[b][: -(-length // page)], device="cuda")
        keys, values = ((codes[at].double() * sc[at].double()[:, :, None, None]).permute(1, 0, 2, 3).reshape(H, -1, D)[:, :length]
                        for codes, sc in ((s["k"], s["ks"]), (s["v"], s["vs"])))
        q = s["q"][starts[b]:starts[b + 1]].double().view(n, H, G, D)
        later = torch.arange(length, device="cuda")[None, :] > torch.arange(length - n, length, device="cuda")[:, None]
        out, lse = torch.empty_like(q), torch.empty((n, H, G), dtype=torch.float64, device="cuda")
        for h in range(H):
            a = torch.einsum("ngd,ld->ngl", q[:, h], keys[h]) / math.sqrt(D)
            a.masked_fill_(later[:, None, :], -math.inf)
            lse[:, h] = torch.logsumexp(a, dim=-1)
            out[:, h] = torch.einsum("ngl,ld->ngd", torch.softmax(a, dim=-1), values[h])
        outs.append(out.reshape(n, H * G, D))
        sums.append(lse.reshape(n, H * G))
    return torch.cat(outs), torch.cat(sums)
