"""Timing cases of the part of a replica's step that goes by its weights, held in 4 bits, and of what it answers with: packing weights,
products with them, the gated half of a feed-forward block, and log probabilities of tokens with entropy and alternatives.

A case is one call (with what belongs to it) of a replica.  ``prepare`` makes what the replica has in hand: packed weights, the
rows of the tokens in the step, logits.  ``run`` makes the call.  The models are those that the roofline is tested with (hidden
4096, 5120 or 8192; feed-forward 14336, 13824 or 28672; 128256 tokens), whole or a device's share of them.

Fields of a case: ``op`` ("pack", "linear", "gated", "logprobs"); ``T`` tokens of the step; ``N`` outputs and ``K`` inputs of a matrix;
``group`` columns that share a pair; ``dtype``; ``pad`` entries by which a row's stride is longer than the row; ``add``: the products
are added to rows that are there (a residual); ``act`` ("silu", "gelu").  For logits: ``V`` tokens in the vocabulary, ``top``
alternatives, ``scale`` (one over the temperature), ``mask``: tokens that are ruled out ("none"; "some": a third of them;
"most": all but a few in every fourth row, and all in one).

Weights in 4 bits: a row is blocks of 128 columns, 16 words of 32 bits each (the last block is filled up).  Word 4 q + m of a block has
the columns 32 m + 8 q + j, j = 0 .. 7, of it: an even j in bits 2 j .. 2 j + 3, an odd one in bits 2 j + 14 .. 2 j + 17.  For each
``group`` columns of a row a pair (step, lo) of the 16-bit type; a code stands for lo + step * code.
"""
import math

import torch

own = False
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _linear(name, T, N, K, group, dtype, add=False, pad=0):
    return dict(name=name, op="linear", T=T, N=N, K=K, group=group, dtype=dtype, add=add, pad=pad)


def _gated(name, T, N, K, group, dtype, act="silu", pad=0):
    return dict(name=name, op="gated", T=T, N=N, K=K, group=group, dtype=dtype, act=act, pad=pad)


def _logprobs(name, T, V, dtype, top, scale=1.0, mask="none", pad=0):
    return dict(name=name, op="logprobs", T=T, V=V, dtype=dtype, top=top, scale=scale, mask=mask, pad=pad)


def listed():
    return [
        # loading a model: a matrix of its attention, and the widest matrix of its feed-forward block, packed and read back
        dict(name="pack_output", op="pack", N=4096, K=4096, group=128, dtype="bf16", pad=0),
        dict(name="pack_gate70", op="pack", N=28672, K=8192, group=64, dtype="fp16", pad=0),
        # a single conversation's step: the output projection with its residual; latency counts
        _linear("linear_one", 1, 4096, 4096, 128, "bf16", add=True),
        # a small replica's step: back from the feed-forward block, onto the residual
        _linear("linear_slots8", 8, 4096, 14336, 64, "bf16", add=True),
        # a full replica's step: queries, keys and values of a large model
        _linear("linear_slots64", 64, 10240, 8192, 128, "fp16"),
        # a prompt's last chunk together with a step of the others: a few hundred rows, an odd number of them
        _linear("linear_chunk", 331, 5120, 13824, 128, "bf16", add=True),
        # a small replica's step into the feed-forward block
        _gated("gated_slots8", 8, 14336, 4096, 128, "bf16"),
        # a full replica's step, a half of a large model's block, small groups
        _gated("gated_slots64", 64, 14336, 8192, 32, "fp16", act="gelu"),
        # prompts that came together, whole: as many rows as their tokens
        _gated("gated_prompts", 4999, 14336, 4096, 128, "bf16"),
        # the answers of a small replica's step
        _logprobs("logprobs_slots8", 8, 128256, "bf16", 5),
        # of a full replica with tokens ruled out and a temperature, from logits in 32 bits
        _logprobs("logprobs_slots64", 64, 128256, "fp32", 20, scale=1.25, mask="most"),
        # of every token of a prompt
        _logprobs("logprobs_prompt", 2311, 128256, "bf16", 8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("pack", "linear", "linear", "linear", "gated", "gated", "logprobs", "logprobs"))
    case = dict(op=op, dtype=rng.choice(("bf16", "bf16", "fp16")), pad=rng.choice((0, 0, 8, 24)))
    if op == "logprobs":
        case.update(dtype=rng.choice(("bf16", "fp16", "fp32")), T=_log(rng, 1, 2311), V=_log(rng, 1000, 128256), top=rng.choice((0, 1, 5, 20, 64)),
                    scale=rng.choice((1.0, 1.0, 0.7, 2.5)), mask=rng.choice(("none", "some", "most")), pad=rng.choice((0, 0, 1, 47)))
        if case["dtype"] == "fp32":
            case["T"] = min(case["T"], 1155)
        return case
    case["group"] = rng.choice((32, 64, 128, 128))
    case["K"] = _log(rng, 256, 14336)
    case["K"] -= case["K"] % rng.choice((8, 128, 128))
    case["N"] = _log(rng, 64, 28672)
    if op == "pack":
        return case
    if op == "linear":
        case["add"] = rng.random() < 0.5
    else:
        case["act"], case["N"] = rng.choice(("silu", "silu", "gelu")), case["N"] // 2
    case["T"] = min(_log(rng, 1, 8192), (1 << 38) // (case["N"] * case["K"]))
    return case


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    made = lambda *shape: torch.randn(shape, generator=gen, device="cuda")     # noqa: E731
    dtype, pad, op = DTYPES[case["dtype"]], case["pad"], case["op"]
    state = dict(case=case)

    def rows(x):                                       # in rows that are `pad` entries longer
        wide = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=dtype, device="cuda")
        wide[:, :x.shape[1]] = x
        return wide[:, :x.shape[1]]

    if op == "logprobs":
        T, V = case["T"], case["V"]
        x = 2.0 * made(T, V)                           # a few tokens stand out, by more in some rows than in others
        x.scatter_add_(1, torch.randint(0, V, (T, 40), generator=gen, device="cuda"), 3.0 * made(T, 40) + 8.0 * torch.rand((T, 1), generator=gen, device="cuda"))
        tokens = torch.where(torch.rand(T, generator=gen, device="cuda") < 0.6, x.argmax(1), torch.randint(0, V, (T,), generator=gen, device="cuda"))
        if case["mask"] == "some":
            x[:, torch.rand(V, generator=gen, device="cuda") < 0.33] = -math.inf
        elif case["mask"] == "most":
            left = torch.randint(0, V, (T, 12), generator=gen, device="cuda")
            kept = x.gather(1, left)
            x[0::4] = -math.inf
            x.scatter_(1, left, kept)
            x[T // 2] = -math.inf
        state["logits"] = rows(x.to(dtype))
        state["tokens"] = torch.where(torch.rand(T, generator=gen, device="cuda") < 0.05, -1, tokens).int()    # no token: -1
        f = lambda *shape, t=torch.float32: torch.zeros(shape, dtype=t, device="cuda")     # noqa: E731
        state["out"] = dict(logprob=f(T), entropy=f(T), ids=f(T, case["top"], t=torch.int32), tops=f(T, case["top"]))
    else:
        N, K, group = case["N"], case["K"], case["group"]
        weights = lambda: made(N, K).mul_(K ** -0.5)   # noqa: E731
        if op == "pack":
            state["values"] = rows(weights())
            blocks = -(-K // 128)
            state["w"] = [(torch.zeros((N, blocks * 16), dtype=torch.int32, device="cuda"),
                           torch.zeros((N, blocks * 128 // group, 2), dtype=dtype, device="cuda"))]
            state["out"] = torch.zeros((N, K), dtype=dtype, device="cuda")
        else:
            state["w"] = [_packed(weights().to(dtype), group) for _ in range(2 if op == "gated" else 1)]
            loud = 1.0 + 7.0 * (torch.rand(K, generator=gen, device="cuda") < 0.005)       # a few channels are louder than others
            state["x"] = rows(made(case["T"], K) * loud + 0.1 * made(K))
            if case.get("add"):
                state["add"] = made(case["T"], N).to(dtype)
            state["out"] = torch.zeros((case["T"], N), dtype=dtype, device="cuda")
    if own:                                            # the descriptions of its memory that a program keeps
        from paper_2604_07144_amd import binding as b
        code = {"bf16": b.AP_BF16, "fp16": b.AP_FP16, "fp32": b.AP_FP32}[case["dtype"]]
        vectors = lambda x: b.make_vectors(x.data_ptr(), x.shape[1], x.stride(0) * x.element_size())           # noqa: E731
        if op == "logprobs":
            x = state["logits"]
            state["d"] = b.make_logits(code, case["T"], case["V"], x.data_ptr(), x.stride(0) * x.element_size())
            need = b.ap_logprobs_workspace(state["d"], case["top"])
        else:
            state["d"] = [b.make_weights(code, case["group"], case["N"], case["K"], c.data_ptr(), p.data_ptr()) for c, p in state["w"]]
            state["d_rows"] = {f: vectors(state[f]) for f in ("x", "add", "out", "values") if f in state}
            need = 0 if op == "pack" else b.ap_linear_workspace(*state["d"], case["T"]) if op == "linear" else b.ap_gated_workspace(*state["d"], case["T"])
        state["space"] = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")
    return state


def run(state):
    case = state["case"]
    if not own:
        return {"pack": _plain_pack, "linear": _plain_linear, "gated": _plain_gated, "logprobs": _plain_logprobs}[case["op"]](state)
    from paper_2604_07144_amd import binding as b
    stream, out, space = torch.cuda.current_stream().cuda_stream, state["out"], state["space"]
    if case["op"] == "logprobs":
        b.ap_logprobs(state["d"], state["tokens"].data_ptr(), case["scale"], case["top"], out["logprob"].data_ptr(), out["entropy"].data_ptr(),
                      out["ids"].data_ptr(), out["tops"].data_ptr(), space.data_ptr(), space.numel(), stream)
        return out
    rows = state["d_rows"]
    if case["op"] == "pack":
        b.ap_weights_pack(state["d"][0], rows["values"], stream)
        b.ap_weights_read(state["d"][0], rows["out"], stream)
    elif case["op"] == "linear":
        b.ap_linear(state["d"][0], rows["x"], rows["out"], case["T"], rows.get("add"), space.data_ptr(), space.numel(), stream)
    else:
        b.ap_gated(*state["d"], rows["x"], rows["out"], case["T"], {"silu": b.AP_SILU, "gelu": b.AP_GELU}[case["act"]], space.data_ptr(), space.numel(), stream)
    return out


def _packed(x, group):
    """Words and pairs of rows in the 16-bit type: the step is rounded up, so that 15 steps reach the largest."""
    N, K = x.shape
    blocks = -(-K // 128)
    wide = torch.nn.functional.pad(x, (0, blocks * 128 - K)).unflatten(1, (-1, group))
    here = (torch.arange(blocks * 128, device="cuda") < K).view(-1, group)     # what fills the last block up is in no group's range
    lo = torch.where(here, wide, math.inf).amin(-1)
    hi = torch.where(here, wide, -math.inf).amax(-1)
    some = here.any(-1)
    lo, hi = torch.where(some, lo, 0.0), torch.where(some, hi, 0.0)
    want = (hi.float() - lo.float()) / torch.full_like(lo, 15.0, dtype=torch.float32)      # a quotient: by a plain number it would be a product
    step = want.to(x.dtype)
    step = torch.where(step.float() < want, (step.view(torch.int16) + 1).view(x.dtype), step)
    there = step.float()[..., None]
    code = (wide.float().sub_(lo.float()[..., None])).div_(torch.where(there > 0, there, 1.0)).round_().clamp_(0, 15).to(torch.int32)
    code = torch.where(here, code, 0).view(N, blocks, 4, 4, 4, 2)              # [block][m][q][pair][odd]
    shift = torch.tensor([[0, 16], [4, 20], [8, 24], [12, 28]], device="cuda", dtype=torch.int32)
    words = (code << shift).sum((-2, -1), dtype=torch.int32)                   # bits of their own each
    return words.transpose(2, 3).reshape(N, blocks * 16).contiguous(), torch.stack([step, lo], -1).contiguous()


def _valued(words, pairs, K):
    """What the codes stand for, in 32 bits."""
    N, group = words.shape[0], words.shape[1] * 8 // pairs.shape[1]
    shift = torch.tensor([[0, 16], [4, 20], [8, 24], [12, 28]], device="cuda", dtype=torch.int32)
    code = words.view(N, -1, 4, 4).transpose(2, 3)[..., None, None] >> shift & 15
    code = code.reshape(N, -1, group).float()
    return code.mul_(pairs[..., :1].float()).add_(pairs[..., 1:].float()).flatten(1)[:, :K]


def _plain_pack(state):
    case, (words, pairs) = state["case"], state["w"][0]
    made = _packed(state["values"], case["group"])
    words.copy_(made[0])
    pairs.copy_(made[1])
    return state["out"].copy_(_valued(words, pairs, case["K"]))


def _plain_linear(state):
    y = state["x"].float() @ _valued(*state["w"][0], state["case"]["K"]).T
    if "add" in state:
        y = state["add"].float() + y
    return state["out"].copy_(y)


def _plain_gated(state):
    x, K = state["x"].float(), state["case"]["K"]
    gate, up = (x @ _valued(*w, K).T for w in state["w"])
    if state["case"]["act"] == "silu":
        gate = gate / (1.0 + torch.exp(-gate))
    else:
        gate = 0.5 * gate * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (gate + 0.044715 * gate * gate * gate)))
    return state["out"].copy_(gate * up)


def _ordered(x):
    """Whole numbers in the order of the values, for values that are numbers."""
    bits = x.view(torch.int16 if x.dtype.itemsize == 2 else torch.int32).long()
    least = -(1 << 8 * x.dtype.itemsize - 1)
    return torch.where(bits < 0, least - bits, bits)   # -0 and 0 are one


def _plain_logprobs(state):
    """Alternatives go by the logits themselves, of equal ones the lowest token first; what is ruled out is none."""
    case, x, tokens, out = state["case"], state["logits"], state["tokens"].long(), state["out"]
    s = x.float() * case["scale"]
    most = s.amax(1, keepdim=True)
    s = s - torch.where(most == -math.inf, 0.0, most)
    e = torch.exp(s)
    total = e.sum(1, dtype=torch.float64)
    log = torch.log(total)
    mean = torch.where(e > 0, e * s, 0.0).sum(1, dtype=torch.float64) / total
    some = total > 0
    out["entropy"].copy_(torch.where(some, log - mean, 0.0))
    given = (tokens >= 0) & (tokens < case["V"])
    of = s.gather(1, torch.where(given, tokens, 0)[:, None])[:, 0].double()
    out["logprob"].copy_(torch.where(given, torch.where(some, of - log, -math.inf), 0.0))
    if case["top"]:
        index = torch.arange(case["V"], device="cuda")
        best = ((_ordered(x) << 32) | ((1 << 32) - 1 - index)).topk(case["top"], 1).values
        ids = ((1 << 32) - 1) - (best & ((1 << 32) - 1))
        of = s.gather(1, ids).double()
        there = of > -math.inf
        out["ids"].copy_(torch.where(there, ids, -1))
        out["tops"].copy_(torch.where(there, of - log[:, None], -math.inf))
    return out


def work(case):
    """Bytes: weights as they are held, rows and logits, once each.  Operations: two for each weight and token; for an entry of the
    logits a comparison, an exponential and two sums."""
    if case["op"] == "logprobs":
        T, V = case["T"], case["V"]
        return {"bytes": T * V * DTYPES[case["dtype"]].itemsize + 12 * T + 8 * T * case["top"], "flops": 5 * T * V}
    N, K = case["N"], case["K"]
    held = N * (K / 2 + 4 * K / case["group"])
    if case["op"] == "pack":
        return {"bytes": int(4 * N * K + 2 * held), "flops": 4 * N * K}
    T, n = case["T"], 2 if case["op"] == "gated" else 1
    return {"bytes": int(n * held + 2 * T * K + 2 * T * N * (2 if case.get("add") else 1)), "flops": 2 * n * T * N * K}


def exact(case, seed):
    """From the definitions, in 64 bits."""
    x = prepare(case, seed)
    if case["op"] == "logprobs":
        V, top = case["V"], case["top"]
        found = dict(logprob=[], entropy=[], ids=[], tops=[])
        for row, token in zip(x["logits"], x["tokens"].tolist()):
            s = row.double() * case["scale"]
            p = torch.softmax(s, 0) if torch.isfinite(s).any() else torch.zeros_like(s)
            logs = s - torch.logsumexp(s, 0) if torch.isfinite(s).any() else s
            kept = torch.nonzero(p > 0)[:, 0]
            found["entropy"].append(-(p[kept] * logs[kept]).sum())
            found["logprob"].append(logs[token] if 0 <= token < V else torch.zeros((), dtype=torch.float64, device="cuda"))
            if top:
                least = torch.topk(row.float(), top).values[-1]
                near = torch.nonzero((row.float() >= least) & (row > -math.inf))[:, 0]     # ascending: a stable sort leaves equal ones so
                near = near[torch.sort(row[near].float(), descending=True, stable=True).indices][:top]
                fill = top - len(near)
                found["ids"].append(torch.nn.functional.pad(near, (0, fill), value=-1).int())
                found["tops"].append(torch.nn.functional.pad(logs[near], (0, fill), value=-math.inf))
        of = {f: torch.stack(r) for f, r in found.items() if r}
        if not top:
            of["ids"], of["tops"] = (torch.zeros((case["T"], 0), dtype=t, device="cuda") for t in (torch.int32, torch.float64))
        return of
    N, K, group, dtype = case["N"], case["K"], case["group"], DTYPES[case["dtype"]]
    if case["op"] == "pack":
        out = torch.empty((N, K), dtype=torch.float64, device="cuda")
        for k in range(0, K, group):                   # the values that the codes of a group stand for
            r = x["values"][:, k:k + group].double()
            lo, hi = r.min(1, keepdim=True).values, r.max(1, keepdim=True).values
            want = (hi - lo) / torch.full_like(lo, 15.0)
            near = want.to(dtype)
            step = (near.view(torch.int16) + (near.double() < want).short()).view(dtype).double()
            out[:, k:k + group] = lo + step * torch.round((r - lo) / torch.where(step > 0, step, 1.0)).clamp(0, 15)
        return out
    c = torch.arange(K, device="cuda")
    j = c % 8
    word, shift = c // 128 * 16 + c % 32 // 8 * 4 + c % 128 // 32, j // 2 * 4 + j % 2 * 16
    products = []
    for words, pairs in x["w"]:
        two = pairs.double()[:, c // group]
        w = two[..., 1] + two[..., 0] * (words[:, word].long() >> shift & 15)
        products.append(x["x"].double() @ w.T)
    if case["op"] == "linear":
        return products[0] + x["add"].double() if "add" in x else products[0]
    gate, up = products
    if case["act"] == "silu":
        return gate * torch.sigmoid(gate) * up
    return 0.5 * gate * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (gate + 0.044715 * gate ** 3))) * up
