"""Operators of a served language model beside an ASER-quantized layer, as cases that can be timed and compared.

A case is a dict of plain values; its "kind" says which operator a pass goes through:

  adapters   low-rank adapters of many requests added to a projection's output: every token names one adapter of a
             pool or none, Y[m] + scale_a B_a (A_a x[m]), each adapter of a rank of its own (AserAdapters.add)
  adapted    a quantized projection together with the adapters of its tokens, in one call (AserLinear.__call__)
  ffn        a gated feed-forward block of quantized layers: H = act(X Wg^T) * (X Wu^T), Y = H Wd^T, with the
             per-token quantization and the low-rank terms of each layer (AserGatedFFN)

A quantized layer is  Y = fp16( a_scale w_scale (Xq Wq^T) + T L_B^T )  with  x~ = x / s,  a_scale = max|x~| / 127,
Xq = clamp(rne(x~ / a_scale), +-127) per token,  T = bf16(x~ L_A^T): the codes, T, a projection's output before its
adapters, the outputs of gate and up and H (fp16) are stored values, and their roundings belong to the definition.
"""
import math

import torch

own = False          # set by the caller: False = the plain forms below, True = the framework's operators


def listed():
    return [
        # one sequence, one new token, one adapter of the usual small rank on an attention projection: the smallest call
        dict(kind="adapters", tokens=1, k=4096, n=4096, rank=16, slots=8, used=1, bare=0.0, mixed=True, name="adapters_decode_1"),
        # a decode step of 64 sequences that use 32 adapters of ranks 64, 32 and 16, a few of them none
        dict(kind="adapters", tokens=64, k=4096, n=4096, rank=64, slots=48, used=32, bare=0.1, mixed=True, name="adapters_decode_64"),
        # a ragged batch of prompt chunks of 8 requests on the fused gate and up projection
        dict(kind="adapters", tokens=501, k=4096, n=28672, rank=32, slots=16, used=8, bare=0.0, mixed=False, name="adapters_chunk_501"),
        # prompts of 6 requests on an attention projection
        dict(kind="adapters", tokens=4096, k=4096, n=4096, rank=64, slots=16, used=6, bare=0.0, mixed=False, name="adapters_prefill_4096"),
        # prompts of 5 requests and some without an adapter, long rows and a high rank: a down projection
        dict(kind="adapters", tokens=2048, k=14336, n=4096, rank=128, slots=8, used=5, bare=0.2, mixed=False, name="adapters_down_2048"),
        # a decode step of 16 sequences, each with an adapter of its own, through a quantized attention projection
        dict(kind="adapted", tokens=16, k=4096, n=4096, rank=16, slots=16, used=16, bare=0.0, mixed=True, base_rank=64, name="adapted_decode_16"),
        # prompts of 4 requests through a quantized attention projection
        dict(kind="adapted", tokens=1024, k=4096, n=4096, rank=32, slots=8, used=4, bare=0.1, mixed=False, base_rank=64, name="adapted_prompt_1024"),
        # one new token through the feed-forward block of an 8B-class model
        dict(kind="ffn", tokens=1, k=4096, f=14336, rank=64, rank_down=64, act="silu", name="ffn_decode_1"),
        # a decode step of 16 sequences
        dict(kind="ffn", tokens=16, k=4096, f=14336, rank=128, rank_down=128, act="silu", name="ffn_decode_16"),
        # a decode step of a full batch through a 70B-class block
        dict(kind="ffn", tokens=64, k=8192, f=28672, rank=32, rank_down=32, act="silu", name="ffn_70b_64"),
        # a ragged chunk of a prompt mixed with running sequences, the activation of another model family
        dict(kind="ffn", tokens=333, k=4096, f=14336, rank=64, rank_down=64, act="gelu_tanh", name="ffn_chunk_333"),
        # prefill of a batch of prompts: the largest call
        dict(kind="ffn", tokens=4096, k=4096, f=14336, rank=128, rank_down=128, act="silu", name="ffn_prefill_4096"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["adapters", "adapters", "adapted", "ffn"])
    tokens = _log(rng, 1, 4096)
    if kind == "ffn":
        k = 128 * _log(rng, 4, 64)
        f = 128 * _log(rng, 4, 112)
        if k * f > 4096 * 14336:
            tokens = min(tokens, 1024)
        return dict(kind=kind, tokens=tokens, k=k, f=f, rank=16 * rng.choice([0, 1, 2, 4, 6, 8, 12]),
                    rank_down=16 * rng.choice([0, 1, 2, 4, 6, 8, 12]), act=rng.choice(["silu", "gelu_tanh"]))
    rank = 16 * rng.choice([1, 1, 2, 2, 3, 4, 4, 6, 8, 16])
    k = 128 * _log(rng, 4, 112)
    n = 8 * _log(rng, 64, 3584 if kind == "adapters" else 1792)
    slots = min(_log(rng, 1, 64), max(1, 100_000_000 // (rank * (k + n))))
    used = min(slots, tokens, _log(rng, 1, 64))
    case = dict(kind=kind, tokens=tokens, k=k, n=n, rank=rank, slots=slots, used=used, bare=rng.choice([0.0, 0.0, 0.1, 0.4]),
                mixed=rng.random() < 0.5)
    if kind == "adapted":
        case["base_rank"] = 16 * rng.choice([0, 2, 4, 8])
    return case


# ----------------------------------------------------------------------------
# what a program has in hand before the call
# ----------------------------------------------------------------------------
class _Maker:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed) & 0x7FFFFFFF)

    def normal(self, *shape, scale=1.0):
        return torch.randn(*shape, device="cuda", dtype=torch.float16, generator=self.g) * scale

    def order(self, n):
        return torch.randperm(n, device="cuda", generator=self.g)


def _ranks(case):
    """The rank of every used adapter: the largest, half and a quarter of it in turn, in steps of 16."""
    return [max(16, (case["rank"] >> (i % 3)) // 16 * 16) for i in range(case["used"])]


def _bare(case):
    return min(int(case["tokens"] * case["bare"]), case["tokens"] - case["used"])


def _adapter_inputs(m, case):
    """The pool A [slots, rank, K], B [slots, N, rank] with a rank and a factor for each adapter, and the adapter of each
    token (-1: none).  Rows of A and columns of B behind an adapter's own rank hold what an earlier tenant left there."""
    tokens, slots, used, r = case["tokens"], case["slots"], case["used"], case["rank"]
    st = {"A": m.normal(slots, r, case["k"], scale=0.02), "B": m.normal(slots, case["n"], r, scale=0.02)}
    chosen = m.order(slots)[:used]
    st["ranks"] = torch.full((slots,), r, device="cuda", dtype=torch.int32)
    st["ranks"][chosen] = torch.tensor(_ranks(case), device="cuda", dtype=torch.int32)
    st["scale"] = 0.5 + torch.rand(slots, device="cuda", generator=m.g)
    bare = _bare(case)
    whose = torch.full((tokens,), -1, device="cuda", dtype=torch.int32)
    # tokens with an adapter: every used one has at least one token; runs of tokens in a batch of prompts
    at = torch.cat([torch.arange(used, device="cuda"),
                    torch.randint(0, used, (tokens - bare - used,), device="cuda", generator=m.g)]).sort().values
    whose[:tokens - bare] = chosen[at].int()
    st["slot"] = whose[m.order(tokens)].contiguous() if case["mixed"] else whose
    return st


def _activations(m, tokens, k, idx, gain=30.0):
    x = m.normal(tokens, k)
    x[:, idx] *= gain
    return x


def _smoothing(x, w, idx):
    s = torch.ones(x.shape[1], device="cuda", dtype=torch.float32)
    s[idx] = (x[:, idx].abs().amax(0).float() / w[:, idx].abs().amax(0).float()).sqrt().clamp_min(1e-3)
    return s


def _factors(m, k, n, rank):
    return (m.normal(rank, k, scale=0.02), m.normal(n, rank, scale=0.02)) if rank else (None, None)


def _inputs(case, seed):
    m = _Maker(seed)
    kind, tokens, k = case["kind"], case["tokens"], case["k"]
    if kind == "adapters":
        st = _adapter_inputs(m, case)
        st["X"] = _activations(m, tokens, k, m.order(k)[:max(1, k // 100)])
        st["Y"] = m.normal(tokens, case["n"])
        return st
    idx = m.order(k)[:max(1, k // 100)]
    x = _activations(m, tokens, k, idx)
    if kind == "adapted":
        st = _adapter_inputs(m, case)
        w = m.normal(case["n"], k, scale=0.02)
        st.update(X=x, W=w, s=_smoothing(x, w, idx))
        st["L_A"], st["L_B"] = _factors(m, k, case["n"], case["base_rank"])
        return st
    f, sigma = case["f"], 0.64 / math.sqrt(k)
    st = {"X": x, "W_gate": m.normal(f, k, scale=sigma), "W_up": m.normal(f, k, scale=sigma),
          "W_down": m.normal(k, f, scale=0.02), "act": case["act"]}
    loud = m.order(f)[:max(1, f // 100)]                    # channels of H with large values, which the down layer smooths
    st["W_up"][loud] *= 8.0
    st["s"] = _smoothing(x, st["W_up"], idx)
    st["s_down"] = torch.ones(f, device="cuda", dtype=torch.float32)
    st["s_down"][loud] = 20.0 + 8.0 * torch.rand(loud.numel(), device="cuda", generator=m.g)
    st["L_A"], st["L_B"] = _factors(m, k, 2 * f, case["rank"])           # L_B: the rows of gate, then those of up
    st["L_A_down"], st["L_B_down"] = _factors(m, f, k, case["rank_down"])
    return st


def _weight_codes(w, s):
    ws = w.float() * s
    scale = ws.abs().amax(1) / 7.0
    q = (ws / torch.where(scale > 0, scale, 1.0)[:, None]).round_().clamp_(-8, 7).to(torch.int8)
    return q, scale


def prepare(case, seed):
    st = _inputs(case, seed)
    st["kind"] = case["kind"]
    tokens = case["tokens"]
    if own:
        import paper_2411_07762_b200 as aser

        if case["kind"] != "ffn":
            # the pool stays from call to call; the plan is made once for a batch and serves every layer of its step
            st["adapters"] = aser.AserAdapters(st["A"], st["B"], scale=st["scale"], ranks=st["ranks"])
            st["plan"] = st["adapters"].plan(st["slot"])
        if case["kind"] == "adapters":
            st["out"] = torch.empty_like(st["Y"])
        elif case["kind"] == "adapted":
            st["layer"] = aser.AserLinear(st.pop("W"), st["s"], st["L_A"], st["L_B"], tokens)
        else:
            st["block"] = aser.AserGatedFFN(st.pop("W_gate"), st.pop("W_up"), st["s"], st["L_A"], st["L_B"], st.pop("W_down"),
                                            st["s_down"], st["L_A_down"], st["L_B_down"], tokens, activation=case["act"])
    elif case["kind"] == "adapted":
        st["Wq"], st["w_scale"] = _weight_codes(st.pop("W"), st["s"])
    elif case["kind"] == "ffn":
        st["Wq"], st["w_scale"] = _weight_codes(torch.cat([st.pop("W_gate"), st.pop("W_up")]), st["s"])
        st["Wq_down"], st["w_scale_down"] = _weight_codes(st.pop("W_down"), st["s_down"])
    return st


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------
def _plain_adapters(st):
    """scale_a B_a (A_a x) in fp32, for every token: the products with all adapters of the pool, of which a token keeps its own."""
    slots, r, k = st["A"].shape
    n = st["B"].shape[1]
    slot = torch.arange(slots, device="cuda")
    down = (st["X"].float() @ st["A"].float().reshape(slots * r, k).T).reshape(-1, slots, r)
    mine = (st["slot"][:, None] == slot[None, :])[:, :, None] & (torch.arange(r, device="cuda")[None, :] < st["ranks"][:, None])[None]
    down = torch.where(mine, down * st["scale"][None, :, None], 0.0)
    return down.reshape(-1, slots * r) @ st["B"].float().permute(0, 2, 1).reshape(slots * r, n)


def _plain_layer(x, s, w_codes, w_scale, l_a, l_b):
    """A quantized layer in fp32, before its output is rounded.  (The integer sums are exact in fp32.)"""
    xs = x.float() / s
    a_scale = xs.abs().amax(1) / 127.0
    q = (xs / torch.where(a_scale > 0, a_scale, 1.0)[:, None]).round().clamp(-127, 127)
    y = (q @ w_codes.float().T) * (a_scale[:, None] * w_scale[None, :])
    if l_a is not None:
        t = (xs @ l_a.float().T).bfloat16().float()
        y = y + t @ l_b.float().T
    return y


def _plain_act(g, act):
    if act == "silu":
        return g / (1.0 + torch.exp(-g))
    return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g * g * g)))


def run(st):
    kind = st["kind"]
    if own:
        if kind == "adapters":
            return st["adapters"].add(st["X"], st["Y"], st["plan"], out=st["out"])
        if kind == "adapted":
            return st["layer"](st["X"], adapters=st["adapters"], plan=st["plan"])
        return st["block"](st["X"])
    if kind == "adapters":
        return (st["Y"].float() + _plain_adapters(st)).half()
    if kind == "adapted":
        return (_plain_layer(st["X"], st["s"], st["Wq"], st["w_scale"], st["L_A"], st["L_B"]).half().float() + _plain_adapters(st)).half()
    g, u = _plain_layer(st["X"], st["s"], st["Wq"], st["w_scale"], st["L_A"], st["L_B"]).half().float().chunk(2, dim=1)
    h = (_plain_act(g, st["act"]) * u).half()
    return _plain_layer(h, st["s_down"], st["Wq_down"], st["w_scale_down"], st["L_A_down"], st["L_B_down"]).half()


# ----------------------------------------------------------------------------
# the same outputs in 64 bits, one adapter and one layer after the other
# ----------------------------------------------------------------------------
def _exact_layer(x, w, s, l_a, l_b):
    x, s = x.double(), s.double()
    xs = x / s
    top = xs.abs().max(dim=1, keepdim=True).values
    codes = torch.clamp(torch.round(xs * 127 / torch.where(top > 0, top, torch.ones_like(top))), -127, 127)
    ws = w.double() * s
    wtop = ws.abs().max(dim=1, keepdim=True).values
    wcodes = torch.clamp(torch.round(ws * 7 / torch.where(wtop > 0, wtop, torch.ones_like(wtop))), -8, 7)
    y = torch.mm(codes * (top / 127), (wcodes * (wtop / 7)).t())
    if l_a is not None:
        y += torch.mm(torch.mm(xs, l_a.double().t()).to(torch.bfloat16).double(), l_b.double().t())
    return y


def exact(case, seed):
    st = _inputs(case, seed)
    if case["kind"] == "ffn":
        gate, up = [_exact_layer(st["X"], st[w], st["s"], st["L_A"], None if st["L_B"] is None else lb).half().double()
                    for w, lb in (("W_gate", None if st["L_B"] is None else st["L_B"][:case["f"]]),
                                  ("W_up", None if st["L_B"] is None else st["L_B"][case["f"]:]))]
        if case["act"] == "silu":
            gate = gate * torch.sigmoid(gate)
        else:                                                  # the tanh form, written with the logistic function
            gate = gate * torch.sigmoid(math.sqrt(8.0 / math.pi) * (gate + 0.044715 * gate ** 3))
        return _exact_layer((gate * up).half(), st["W_down"], st["s_down"], st["L_A_down"], st["L_B_down"])
    if case["kind"] == "adapters":
        y = st["Y"].double()
    else:
        y = _exact_layer(st["X"], st["W"], st["s"], st["L_A"], st["L_B"]).half().double()
    ranks, slots = st["ranks"].tolist(), st["slot"].tolist()
    for a in sorted(set(slots) - {-1}):
        rows = (st["slot"] == a).nonzero().flatten()
        r = ranks[a]
        y[rows] += float(st["scale"][a]) * torch.mm(torch.mm(st["X"][rows].double(), st["A"][a, :r].double().t()), st["B"][a, :, :r].double().t())
    return y


# ----------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------
def _layer_work(tokens, k, n, rank):
    b = 4 * k + 2 * rank * k + n * k // 2 + 4 * n + 2 * n * rank
    return b, 2 * tokens * k * n + 2 * tokens * rank * (k + n)


def work(case):
    tokens, k = case["tokens"], case["k"]
    if case["kind"] == "ffn":
        b1, f1 = _layer_work(tokens, k, 2 * case["f"], case["rank"])
        b2, f2 = _layer_work(tokens, case["f"], k, case["rank_down"])
        return {"bytes": b1 + b2 + 4 * tokens * k, "flops": f1 + f2 + 8 * tokens * case["f"]}
    n, ranks = case["n"], _ranks(case)
    adapted = tokens - _bare(case)
    mean = sum(ranks) / len(ranks)
    flops = 2 * adapted * mean * (k + n)
    b = 2 * sum(ranks) * (k + n) + 4 * tokens + 8 * case["slots"]
    if case["kind"] == "adapters":
        return {"bytes": b + 2 * adapted * k + 4 * tokens * n, "flops": flops}
    lb, lf = _layer_work(tokens, k, n, case["base_rank"])
    return {"bytes": b + lb + 2 * tokens * (k + n), "flops": flops + lf}
