"""The products around the routing call whose speed counts, as a program that serves a
mixture-of-experts model makes them: sizes, inputs, one pass in plain form and through the
library, the definition in 64 bits, and the work a pass cannot do without.

Three operators ("op" of a case):

  up       the experts' first product over the routing tables: gathered rows, gate and up
           matrix of each expert, silu(gate) * up
  down     the experts' second product: back to token order, weighted, summed over a token's
           experts, with or without a residual input
  adapted  a projection that all rows share, and beside it the low-rank adapters that the
           requests of the batch bring along

Routing tables are made like the ones of the routing call: each token has k distinct experts
whose popularity falls like rank^-1.1 under a rank map of the layer ("zipf"), or is even, and
the assignments are grouped by expert in ascending order.  A case may hold a share of the
experts only (first, E of total), as one of several GPUs does.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _experts(name, op, T, H, F, E, k, dtype="bf16", total=None, first=0, skew=1.1, base=False):
    return dict(name=name, op=op, T=T, H=H, F=F, E=E, k=k, dtype=dtype, total=E if total is None else total,
                first=first, skew=skew, base=base)


def _adapted(name, T, H, N, R, M, requests, dtype="bf16", out="bf16", bare=0.0, one_each=False):
    return dict(name=name, op="adapted", T=T, H=H, N=N, R=R, M=M, requests=requests, dtype=dtype, out=out,
                bare=bare, one_each=one_each)


def listed():
    return [
        # One sequence being decoded: one token, its six experts, each with a single row.
        _experts("up_one_token", "up", 1, 2048, 1408, 64, 6),
        # A decode step of 64 sequences: a few rows for each expert, the weights are the traffic.
        _experts("up_decode", "up", 64, 2048, 1408, 64, 6),
        # A prefill batch of the 64-expert layer, popularity as skewed as the routing benchmark's.
        _experts("up_prefill", "up", 16384, 2048, 1408, 64, 6),
        # The 8-expert layer with wide experts, a chunk of a prompt.
        _experts("up_wide", "up", 4096, 4096, 14336, 8, 2, skew=0.3),
        # Odd sizes in single precision: an odd number of experts, rows and columns that fill no tile.
        _experts("up_odd_f32", "up", 333, 516, 212, 33, 3, dtype="f32"),
        # The second product of the single token, on a residual stream.
        _experts("down_one_token", "down", 1, 2048, 1408, 64, 6, base=True),
        # ... of the decode step of the 8-expert layer: 16 sequences.
        _experts("down_decode_wide", "down", 16, 4096, 14336, 8, 2, skew=0.3, base=True),
        # ... of the prefill batch.
        _experts("down_prefill", "down", 16384, 2048, 1408, 64, 6, base=True),
        # One of four GPUs: 16 of 64 experts, a mid-sized batch of an odd number of tokens.
        _experts("down_share", "down", 1501, 2048, 1408, 16, 6, total=64, first=16),
        # The gate of a decode step whose 64 requests bring 32 adapters of rank 16: fp32 logits.
        _adapted("gate_decode", 64, 2048, 64, 16, 32, 64, out="f32", one_each=True),
        # The gate of a prefill batch of 24 prompts, a few of them without an adapter.
        _adapted("gate_prefill", 16384, 2048, 64, 16, 8, 24, out="f32", bare=0.2),
        # A square projection of a prompt chunk, rank 64, requests that end anywhere.
        _adapted("square_prefill", 4096, 4096, 4096, 64, 16, 19, bare=0.1),
    ]


def _log(rng, lo, hi, step=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    return min(max(v, -(-lo // step) * step), hi // step * step)


def draw(rng):
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    step = 4 if dtype == "f32" else 8
    most = 1.9e12 if dtype == "bf16" else 5e10
    while True:
        if rng.random() < 0.67:
            total = rng.randint(1, 64)
            share = rng.random() < 0.25 and total > 1
            E = rng.randint(1, total) if share else total
            case = _experts(None, rng.choice(["up", "down"]), _log(rng, 1, 16384), _log(rng, 128, 4096, step),
                            _log(rng, 64, 14336, step), E, rng.randint(1, min(total, 8)), dtype=dtype, total=total,
                            first=rng.randint(0, total - E), skew=rng.choice([0.0, 0.3, 1.1]),
                            base=rng.random() < 0.5)
            held = case["E"] * case["F"] * case["H"]
        else:
            T = _log(rng, 1, 16384)
            requests = _log(rng, 1, min(T, 256))
            case = _adapted(None, T, _log(rng, 128, 4096, step), _log(rng, 8, 4096), _log(rng, 8, 128, 8),
                            _log(rng, 1, 64), requests, dtype=dtype, out=rng.choice([dtype, "f32"]),
                            bare=rng.choice([0.0, 0.2]), one_each=requests == T)
            held = 0
        if work(case)["flops"] <= most and held <= 5e8:
            del case["name"]
            return case


def _routing(case, g, dev):
    """ids [T,k] (best first), weights, permutation, offsets of the whole layer."""
    T, k, total = case["T"], case["k"], case["total"]
    rank = torch.randperm(total, generator=g, device=dev)
    bias = -case["skew"] * torch.log(rank.float() + 1)
    noise = -torch.log(-torch.log(torch.rand(T, total, generator=g, device=dev).clamp(1e-9, 1 - 1e-7)))
    score = bias + noise
    top, ids = torch.topk(score, k, dim=1)
    weights = torch.softmax(top, 1)
    flat = ids.reshape(-1)
    order = torch.sort(flat, stable=True)[1]
    counts = torch.bincount(flat, minlength=total)
    offsets = torch.zeros(total + 1, dtype=torch.int32, device=dev)
    offsets[1:] = torch.cumsum(counts, 0).int()
    return ids.int().contiguous(), weights.contiguous(), order.int().contiguous(), offsets


def _inputs(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    t = _TYPES[case["dtype"]]
    T, H = case["T"], case["H"]
    s = dict(case=case)

    def normal(*shape, std):
        out = torch.empty(*shape, dtype=t, device=dev)
        return out.normal_(0.0, std, generator=g)

    if case["op"] in ("up", "down"):
        F, E, k = case["F"], case["E"], case["k"]
        s["ids"], s["weights"], s["permutation"], s["offsets"] = _routing(case, g, dev)
        if case["op"] == "up":
            s["hidden"] = normal(T, H, std=1.0)
            s["w"] = normal(E, 2 * F, H, std=1.5 / math.sqrt(H))
            s["act"] = torch.zeros(T * k, F, dtype=t, device=dev)
        else:
            gate, up = normal(T * k, F, std=1.5), normal(T * k, F, std=1.5)
            s["act"] = (gate.float() * torch.sigmoid(gate.float()) * up.float()).to(t)
            s["w"] = normal(E, H, F, std=1.0 / math.sqrt(F))
            s["base"] = normal(T, H, std=1.0) if case["base"] else None
            s["out"] = torch.empty(T, H, dtype=t, device=dev)
    else:
        N, R, M, n = case["N"], case["R"], case["M"], case["requests"]
        s["x"] = normal(T, H, std=1.0)
        s["w"] = normal(N, H, std=0.02)
        s["a_down"] = normal(M, R, H, std=1.0 / math.sqrt(H))
        s["a_up"] = normal(M, N, R, std=0.1)
        s["scales"] = torch.rand(M, generator=g, device=dev) * 2
        if case["one_each"]:
            cuts = torch.arange(n + 1, device=dev)
        else:  # prompts that end anywhere; two that end at the same row leave an empty one between
            cuts = torch.sort(torch.randint(0, T + 1, (n + 1,), generator=g, device=dev))[0]
            cuts[0], cuts[-1] = 0, T
        s["request_offsets"] = cuts.int().contiguous()
        which = torch.randint(0, M, (n,), generator=g, device=dev)
        none = torch.rand(n, generator=g, device=dev) < case["bare"]
        s["request_adapters"] = torch.where(none, -1, which).int().contiguous()
        s["out"] = torch.empty(T, N, dtype=_TYPES[case["out"]], device=dev)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:  # the parameters and the workspace, which a program makes once for calls of one size
        T, H = case["T"], case["H"]
        from paper_2510_03293_amd import binding as B
        code = {"bf16": B.DTYPE_BF16, "f32": B.DTYPE_F32}
        if case["op"] == "adapted":
            s["params"] = B.make_adapter_params(case["R"], case["M"], case["requests"], dtype=code[case["dtype"]],
                                                out_dtype=code[case["out"]])
            nbytes = B.laser_project_workspace_bytes(T, H, case["N"], s["params"])
        else:
            s["params"] = B.make_experts_params(case["k"], dtype=code[case["dtype"]], first_expert=case["first"])
            nbytes = B.laser_experts_workspace_bytes(T, H, case["F"], case["E"], s["params"])
        s["workspace"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return s


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2510_03293_amd import binding as B
    c = s["case"]
    if c["op"] == "up":
        B.laser_experts_up(s["hidden"], s["w"], c["T"], c["H"], c["F"], c["E"], s["params"], s["permutation"],
                           s["offsets"], s["act"])
        return s["act"]
    if c["op"] == "down":
        B.laser_experts_down(s["act"], s["w"], c["T"], c["H"], c["F"], c["E"], s["params"], s["permutation"],
                             s["offsets"], s["ids"], s["weights"], s["base"], s["out"], s["workspace"])
        return s["out"]
    B.laser_project_adapted(s["x"], s["w"], c["T"], c["H"], c["N"], s["params"], s["a_down"], s["a_up"], s["scales"],
                            s["request_offsets"], s["request_adapters"], s["out"], s["workspace"])
    return s["out"]


def _plain(s):
    c = s["case"]
    if c["op"] == "adapted":
        x = s["x"].float()
        y = x @ s["w"].float().t()
        cuts, which = s["request_offsets"].tolist(), s["request_adapters"].tolist()
        for r, m in enumerate(which):
            a, b = cuts[r], cuts[r + 1]
            if 0 <= m < c["M"] and a < b:
                v = x[a:b] @ s["a_down"][m].float().t()
                y[a:b] += s["scales"][m] * (v @ s["a_up"][m].float().t())
        return y.to(s["out"].dtype)
    F, E, k, first = c["F"], c["E"], c["k"], c["first"]
    cuts = s["offsets"].tolist()
    if c["op"] == "up":
        act = torch.zeros_like(s["act"])
        for e in range(E):
            a, b = cuts[first + e], cuts[first + e + 1]
            if a < b:
                z = s["hidden"][s["permutation"][a:b].long() // k].float() @ s["w"][e].float().t()
                gate, up = z[:, :F], z[:, F:]
                act[a:b] = (gate / (1 + torch.exp(-gate)) * up).to(act.dtype)
        return act
    T, H = c["T"], c["H"]
    y = torch.zeros(T * k, H, device=s["act"].device)
    for e in range(E):
        a, b = cuts[first + e], cuts[first + e + 1]
        if a < b:
            slots = s["permutation"][a:b].long()
            y[slots] = (s["act"][a:b].float() @ s["w"][e].float().t()) * s["weights"].reshape(-1)[slots, None]
    y = y.reshape(T, k, H).sum(1)
    if s["base"] is not None:
        y = y + s["base"].float()
    return y.to(s["out"].dtype)


def _sizes(case):
    """Bytes of one value, positions of the case's experts, experts that are expected to have a row."""
    size = 2 if case["dtype"] == "bf16" else 4
    share = case["E"] / case["total"]
    rows = case["T"] * case["k"] * share
    busy = case["E"] * (1 - (1 - case["k"] / case["total"]) ** case["T"])
    return size, rows, busy


def work(case):
    T, H = case["T"], case["H"]
    if case["op"] == "adapted":
        size = 2 if case["dtype"] == "bf16" else 4
        osize = 2 if case["out"] == "bf16" else 4
        N, R, M = case["N"], case["R"], case["M"]
        used = M * (1 - (1 - 1 / M) ** (case["requests"] * (1 - case["bare"])))
        adapted = T * (1 - case["bare"])
        return {"bytes": int(size * (T * H + N * H + used * R * (H + N)) + osize * T * N),
                "flops": int(2 * T * N * H + 2 * adapted * R * (H + N))}
    F, k = case["F"], case["k"]
    size, rows, busy = _sizes(case)
    if case["op"] == "up":
        return {"bytes": int(size * (min(T, rows) * H + busy * 2 * F * H + rows * F) + 4 * rows),
                "flops": int(4 * rows * F * H)}
    return {"bytes": int(size * (rows * F + busy * F * H + T * H * (2 if case["base"] else 1)) + 12 * T * k),
            "flops": int(2 * rows * F * H)}


def exact(case, seed):
    """The definition in 64 bits: every row on its own terms, blocks of rows to bound the memory."""
    s = _inputs(case, seed)
    dev = s["w"].device
    f64 = torch.float64
    if case["op"] == "adapted":
        T, M = case["T"], case["M"]
        owner = torch.full((T,), -1, dtype=torch.long, device=dev)
        for r in range(case["requests"]):
            owner[int(s["request_offsets"][r]):int(s["request_offsets"][r + 1])] = int(s["request_adapters"][r])
        y = torch.matmul(s["x"].to(f64), s["w"].to(f64).transpose(0, 1))
        for m in range(M):
            rows = torch.nonzero(owner == m)[:, 0]
            if rows.numel():
                delta = s["a_up"][m].to(f64).matmul(s["a_down"][m].to(f64))
                y[rows] += s["scales"][m].to(f64) * s["x"][rows].to(f64).matmul(delta.transpose(0, 1))
        return y
    T, H, F, k, E, first = (case[n] for n in ("T", "H", "F", "k", "E", "first"))
    expert = s["ids"].reshape(-1).long() - first          # by slot
    at = torch.empty(T * k, dtype=torch.long, device=dev)  # position of a slot
    at[s["permutation"].long()] = torch.arange(T * k, device=dev)
    if case["op"] == "up":
        out = torch.zeros(T * k, F, dtype=f64, device=dev)
    else:
        out = torch.zeros(T, H, dtype=f64, device=dev)
        if s["base"] is not None:
            out += s["base"].to(f64)
    for e in range(E):
        every = torch.nonzero(expert == e)[:, 0]
        if not every.numel():
            continue
        w = s["w"][e].to(f64)
        for slots in every.split(4096):
            if case["op"] == "up":
                x = s["hidden"][slots // k].to(f64)
                gate, up = torch.matmul(x, w[:F].t()), torch.matmul(x, w[F:].t())
                out[at[slots]] = gate * torch.sigmoid(gate) * up
            else:
                z = torch.matmul(s["act"][at[slots]].to(f64), w.t())
                out.index_add_(0, slots // k, z * s["weights"].reshape(-1)[slots].to(f64)[:, None])
    return out
