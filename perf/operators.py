"""Layers of compressed sequence models, as cases that can be timed and compared.

A case is a dict of plain values; `listed()` gives the fixed ones, `draw(rng)` one more of the same
ranges.  `run` makes one pass: where the module's `own` is true through this library's public entry
points, else through elementary torch operations in 32 bits that say what the layer is.

Three kinds of case ("op"):
  q4      a fully connected layer with 4-bit weights and one scale per group of inputs (cadnn_q4_fc)
  conv    a short causal depthwise convolution over packed sequences, with the kept tail of each
          sequence (cadnn_causal_conv1d)
  scan    a selective state space scan over packed sequences, with the kept state of each sequence
          (cadnn_selective_scan)
"""
from __future__ import annotations

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16}


def _q4(dtype, n, cin, cout, group, relu):
    return {"op": "q4", "dtype": dtype, "n": n, "cin": cin, "cout": cout, "group": group, "relu": relu}


def _conv(dtype, seqs, tokens, channels, taps, ragged):
    return {"op": "conv", "dtype": dtype, "seqs": seqs, "tokens": tokens, "channels": channels, "taps": taps, "ragged": ragged}


def _scan(dtype, seqs, tokens, channels, dstate, groups, gate, ragged):
    return {"op": "scan", "dtype": dtype, "seqs": seqs, "tokens": tokens, "channels": channels, "dstate": dstate,
            "groups": groups, "gate": gate, "ragged": ragged}


def listed():
    def named(name, case):
        return dict({"name": name}, **case)

    return [
        # the classifier of the benchmark network on one image: the smallest call, where the launch counts
        named("q4-classifier-f32", _q4("f32", 1, 2048, 1000, 64, False)),
        # one new token through a wide projection: all of the weights for one vector
        named("q4-token-f16", _q4("f16", 1, 8192, 8192, 128, False)),
        # the first fully connected layer behind a large feature map, three images, the finest groups
        named("q4-features-f32", _q4("f32", 3, 25088, 4096, 32, True)),
        # a small batch of tokens, sizes that no tile divides
        named("q4-few-odd-f16", _q4("f16", 13, 5003, 4099, 32, False)),
        # a prompt: matrix-core work
        named("q4-prompt-f16", _q4("f16", 2048, 4096, 8192, 128, False)),
        # a prompt in fp32 storage, sizes that no tile divides
        named("q4-prompt-odd-f32", _q4("f32", 777, 2500, 3001, 64, False)),
        # one long prompt through the short convolution: memory traffic and nothing else
        named("conv-prompt-f16", _conv("f16", 1, 8192, 4096, 4, False)),
        # one new token of each of 48 sequences: the kept tails count
        named("conv-tokens-f32", _conv("f32", 48, 48, 2048, 4, False)),
        # one long prompt through the scan: few independent channels, a long axis
        named("scan-prompt-f16", _scan("f16", 1, 4096, 2048, 16, 1, True, False)),
        # nine prompts of different lengths, wide states, channels in groups, no gate
        named("scan-ragged-f32", _scan("f32", 9, 1501, 1000, 64, 4, False, True)),
        # one new token of each of 64 sequences: the states are read and written once
        named("scan-tokens-f16", _scan("f16", 64, 64, 4096, 16, 1, True, False)),
        # one new token of one sequence: latency
        named("scan-token-f32", _scan("f32", 1, 1, 1536, 16, 1, True, False)),
    ]


def _log(rng, lo, hi):
    """An integer in [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(float(lo) * (float(hi) / lo) ** rng.random()))))


def _even(rng, v, step):
    """`v`, half of the time cut to a multiple of `step`."""
    return v if v < step or rng.random() < 0.5 else v - v % step


def draw(rng):
    dtype = rng.choice(["f32", "f16"])
    op = rng.choice(["q4", "q4", "q4", "conv", "scan", "scan"])
    if op == "q4":
        cin, cout = _even(rng, _log(rng, 64, 16384), 128), _even(rng, _log(rng, 64, 16384), 64)
        n = 1 if rng.random() < 0.25 else _log(rng, 1, 2048)
        n = max(1, min(n, 2048 * 4096 * 8192 // (cin * cout) // (1 if dtype == "f16" else 4)))
        return _q4(dtype, n, cin, cout, rng.choice([32, 64, 128]), rng.random() < 0.3)
    seqs = 1 if rng.random() < 0.3 else _log(rng, 2, 64)
    channels = _even(rng, _log(rng, 64, 4096), 64)
    ragged = seqs > 1 and rng.random() < 0.5
    each = 1 if rng.random() < 0.3 else _log(rng, 2, 4096)
    if op == "conv":
        tokens = seqs * max(1, min(each, 8192 * 2048 // (seqs * channels)))
        return _conv(dtype, seqs, tokens, channels, rng.randint(2, 6), ragged)
    dstate = rng.choice([8, 16, 16, 16, 32, 64, 128, rng.randint(1, 80)])
    groups = rng.choice([1, 1, 2, 4])
    channels -= channels % groups
    tokens = seqs * max(1, min(each, 4096 * 2048 * 16 // (seqs * channels * dstate)))
    return _scan(dtype, seqs, tokens, channels, dstate, groups, rng.random() < 0.6, ragged)


def _inputs(case, seed):
    """Everything both forms start from, on the GPU, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = _TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    if case["op"] == "q4":
        cin, cout, group = case["cin"], case["cout"], case["group"]
        groups = -(-cin // group)
        scales = ((0.5 + uniform(cout, groups)) * (0.4 / cin ** 0.5)).to(t).float()     # (what the storage type holds)
        return {"codes": (normal(cout, cin) * 2.7).round().clamp(-8, 7).to(torch.int8), "scales": scales,
                "x": normal(case["n"], cin).to(t), "bias": normal(cout) * 0.1}
    seqs, tokens, channels = case["seqs"], case["tokens"], case["channels"]
    if case["ragged"]:
        cuts = torch.randint(0, tokens + 1, (seqs - 1,), generator=torch.Generator().manual_seed(seed)).sort().values.tolist()
        starts = [0] + cuts + [tokens]
    else:
        starts = [i * (tokens // seqs) for i in range(seqs + 1)]
    s = {"starts": torch.tensor(starts, dtype=torch.int32, device="cuda"), "x": normal(tokens, channels).to(t),
         "longest": max(b - a for a, b in zip(starts, starts[1:]))}
    if case["op"] == "conv":
        k = case["taps"]
        s["w"] = ((uniform(channels, k) * 2 - 1) / k ** 0.5).to(t).float()
        s["bias"] = normal(channels) * 0.1
        s["state"] = normal(seqs, k - 1, channels).to(t)
        return s
    n, groups = case["dstate"], case["groups"]
    steps = torch.exp(uniform(channels) * 4.6 - 6.9)                      # time steps from 0.001 to 0.1
    s["dt_bias"] = torch.log(torch.expm1(steps))
    s["dt"] = (normal(tokens, channels) * 0.7).to(t)
    s["a"] = -torch.arange(1, n + 1, device="cuda", dtype=torch.float32).repeat(channels, 1) * (0.5 + uniform(channels, n))
    s["b"], s["c"] = normal(tokens, groups, n).to(t), normal(tokens, groups, n).to(t)
    s["d"] = normal(channels)
    s["z"] = normal(tokens, channels).to(t) if case["gate"] else None
    s["state"] = normal(seqs, channels, n)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own and case["op"] != "scan":        # the weights, packed once for all calls
        import paper_1905_00571_amd as cad
        dtype = cad.F16 if case["dtype"] == "f16" else cad.F32
        if case["op"] == "q4":
            s["handle"] = cad.cadnn_q4_pack_codes(s["codes"].cpu().numpy(), s["scales"].cpu().numpy(), case["group"], dtype)
            cad.cadnn_q4_prepare(s["handle"])
        else:
            s["handle"] = cad.cadnn_pack_weights(s["w"].cpu().numpy().reshape(case["channels"], 1, 1, case["taps"]), dtype)
            cad.cadnn_depthwise_prepare(s["handle"])
    return s


def _silu(v):
    return v / (1 + torch.exp(-v))


def _plain_q4(s, case):
    spread = s["scales"].repeat_interleave(case["group"], 1)[:, :case["cin"]]
    y = torch.mm(s["x"].float(), (s["codes"].float() * spread).t()) + s["bias"]
    return (y.clamp(min=0) if case["relu"] else y).to(s["x"].dtype)


def _plain_conv(s, case):
    k, tokens, seqs = case["taps"], case["tokens"], case["seqs"]
    starts = s["starts"].long()
    lens = starts[1:] - starts[:-1]
    seq = torch.repeat_interleave(torch.arange(seqs, device="cuda"), lens, output_size=tokens)
    x, tail = s["x"].float(), s["state"].float()
    back = k - 1 - torch.arange(k, device="cuda")                         # tokens that a tap looks back
    place = (torch.arange(tokens, device="cuda") - starts[seq])[:, None] - back
    rows = (torch.arange(tokens, device="cuda")[:, None] - back).clamp(min=0)
    taps = torch.where((place >= 0)[:, :, None], x[rows], tail[seq[:, None], (place + k - 1).clamp(max=k - 2)])
    y = _silu((taps * s["w"].t()).sum(1) + s["bias"]).to(s["x"].dtype)
    place = lens[:, None] - (k - 1) + torch.arange(k - 1, device="cuda")   # of the new tail's rows
    rows = (starts[:-1, None] + place).clamp(0, tokens - 1)
    ids = torch.arange(seqs, device="cuda")[:, None]
    s["state"].copy_(torch.where((place >= 0)[:, :, None], x[rows], tail[ids, (place + k - 1).clamp(max=k - 2)]))
    return {"y": y, "state": s["state"]}


def _plain_scan(s, case):
    """The recurrence h = p * h + q, whose prefixes are joined pairwise at doubling distances."""
    tokens, channels, n = case["tokens"], case["channels"], case["dstate"]
    starts = s["starts"].long()
    lens = starts[1:] - starts[:-1]
    some = lens > 0
    first, last = starts[:-1].clamp(max=tokens - 1), (starts[1:] - 1).clamp(min=0)
    x, dt = s["x"].float(), s["dt"].float() + s["dt_bias"]
    dt = dt.clamp(min=0) + torch.log1p(torch.exp(-dt.abs()))
    per = channels // case["groups"]
    b, c = (s[v].float().repeat_interleave(per, 1) for v in "bc")
    p = torch.exp(dt[:, :, None] * s["a"])
    q = (dt * x)[:, :, None] * b
    # a sequence starts from its own state, whatever lies before it
    began = torch.zeros(tokens, dtype=torch.bool, device="cuda").index_fill_(0, first[some], True)
    q.index_add_(0, first[some], p[first[some]] * s["state"][some])
    p = p * (~began)[:, None, None]
    far = 1
    while far < s["longest"]:
        q = torch.cat([q[:far], q[far:] + p[far:] * q[:-far]])
        p = torch.cat([p[:far], p[far:] * p[:-far]])
        far *= 2
    y = (q * c).sum(2) + s["d"] * x
    if s["z"] is not None:
        y = y * _silu(s["z"].float())
    s["state"].copy_(torch.where(some[:, None, None], q[last], s["state"]))
    return {"y": y.to(s["x"].dtype), "state": s["state"]}


def run(state):
    case = state["case"]
    if own:
        import paper_1905_00571_amd as cad
        if case["op"] == "q4":
            return cad.cadnn_q4_fc(state["handle"], state["x"], state["bias"], cad.ACT_RELU if case["relu"] else cad.ACT_NONE)
        starts = state["starts"] if case["ragged"] else None
        if case["op"] == "conv":
            y = cad.cadnn_causal_conv1d(state["handle"], state["x"], state["state"], starts, case["seqs"], state["bias"], cad.ACT_SILU)
        else:
            y = cad.cadnn_selective_scan(state["x"], state["dt"], state["a"], state["b"], state["c"], d=state["d"], z=state["z"],
                                         dt_bias=state["dt_bias"], softplus=True, state=state["state"], seq_start=starts,
                                         seqs=case["seqs"])
        return {"y": y, "state": state["state"]}
    return {"q4": _plain_q4, "conv": _plain_conv, "scan": _plain_scan}[case["op"]](state, case)


def work(case):
    e = 2 if case["dtype"] == "f16" else 4
    if case["op"] == "q4":
        n, cin, cout = case["n"], case["cin"], case["cout"]
        return {"bytes": cout * cin / 2 + cout * -(-cin // case["group"]) * e + n * (cin + cout) * e + cout * 4,
                "flops": 2 * n * cin * cout}
    seqs, tokens, channels = case["seqs"], case["tokens"], case["channels"]
    if case["op"] == "conv":
        k = case["taps"]
        return {"bytes": 2 * tokens * channels * e + 2 * seqs * (k - 1) * channels * e + channels * (k + 1) * 4,
                "flops": 2 * tokens * channels * (k + 2)}
    n = case["dstate"]
    return {"bytes": ((4 if case["gate"] else 3) * tokens * channels + 2 * tokens * case["groups"] * n) * e
            + (2 * seqs * channels * n + channels * (n + 2)) * 4,
            "flops": tokens * channels * (7 * n + 8)}


def exact(case, seed):
    """The definitions in 64 bits: one dot product per output, one token after the other."""
    s = _inputs(case, seed)
    f = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if case["op"] == "q4":
        if case["n"] * case["cin"] * case["cout"] > 2 ** 38:
            return None
        y = f["bias"].repeat(case["n"], 1)
        group = case["group"]
        for i in range(f["scales"].shape[1]):
            at = slice(i * group, min((i + 1) * group, case["cin"]))
            y += torch.mm(f["x"][:, at], s["codes"][:, at].double().t().contiguous()) * f["scales"][:, i]
        return torch.relu(y) if case["relu"] else y
    starts = s["starts"].tolist()
    y = torch.empty_like(f["x"])
    if case["op"] == "conv":
        k = case["taps"]
        for i, (lo, hi) in enumerate(zip(starts, starts[1:])):
            line = torch.cat([f["state"][i], f["x"][lo:hi]])
            total = f["bias"] + sum(line[j:j + hi - lo] * f["w"][:, j] for j in range(k))
            y[lo:hi] = total * torch.sigmoid(total)
            f["state"][i] = line[line.shape[0] - (k - 1):].clone()
        return {"y": y, "state": f["state"]}
    per = case["channels"] // case["groups"]
    dt = torch.nn.functional.softplus(f["dt"] + f["dt_bias"], threshold=700.0)
    lo, hi = s["starts"][:-1].long(), s["starts"][1:].long()
    for t in range(s["longest"]):          # the t-th token of every sequence that has one
        i = torch.nonzero(lo + t < hi).flatten() if case["ragged"] else slice(None)
        at = lo[i] + t
        b, c = (f[v][at].repeat_interleave(per, 1) for v in "bc")
        h = torch.exp(dt[at][:, :, None] * f["a"]) * f["state"][i] + (dt[at] * f["x"][at])[:, :, None] * b
        f["state"][i] = h
        y[at] = (h * c).sum(2)
    y += f["d"] * f["x"]
    if s["z"] is not None:
        y *= f["z"] * torch.sigmoid(f["z"])
    return {"y": y, "state": f["state"]}
