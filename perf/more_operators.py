"""The 4-bit cache of a serving program as measurable cases, each in a plain form and as the framework's call.

append  The new tokens' keys and values go into paged pools of 4 bits: the 32 elements x of a block (of one
        token's head) share a scale s = 2^e, the least with A < 7 s for their largest magnitude A (e from -124
        to 125), and each is held as the E2M1 code (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) nearest to
        x / s, ties to the even code, saturated at 6. Where the projections come without their position the keys
        are rotated first, pairs (j, j + R/2) or (2j, 2j + 1) by the caller's table of (cos, sin), rounded once to
        32 bits, and the queries are rotated into an output of their own.
read    Rows of the tokens that a pool holds: the keys and values at given positions of every request, as bf16
        rows in the order that the append takes. Pools of 4 bits, of E4M3 codes with one scale each ("fp8"),
        of bf16.
attend  Attention of the new tokens over all that the 4-bit pools hold of their request,
            o = sum_{j <= P_r + i} softmax_j(scale <q, k_j>) v_j      for new token i behind P_r cached ones.
step    append with rotation, then attend with the rotated queries: one layer of a step.

Head shapes are those of the workloads module's Llama-3 models (8B: 32 query and 8 KV heads, 70B: 64 and 8,
head_dim 128), of one GPU's share of the 70B model under tensor parallelism (8 and 1), and head_dim 64 shapes of
the tests.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
K_SCALE, V_SCALE = 0.0123, 0.0119   # 8-bit pools: about 5.4 standard deviations at code 448
BASE = 500000.0                     # rotary base of the Llama-3 models


def listed():
    return [
        # one interactive user's next token at a far position: latency alone
        dict(name="append_one_far", op="append", q_heads=64, kv_heads=8, head_dim=128, rotary=128, pairs="halves",
             fused_qkv=True, batch=1, prefix=65531, spread=0.0, new=1, lengths_seed=1),
        # the next token of 96 conversations
        dict(name="append_decode", op="append", q_heads=64, kv_heads=8, head_dim=128, rotary=128, pairs="interleaved",
             fused_qkv=True, batch=96, prefix=2048, spread=0.8, new=1, lengths_seed=2),
        # contexts that come back from the host tier as rows, a small model
        dict(name="append_contexts_d64", op="append", q_heads=32, kv_heads=8, head_dim=64, rotary=0, pairs="halves",
             fused_qkv=False, batch=16, prefix=0, spread=0.0, new=2003, lengths_seed=4),
        # a long prompt batch of the 70B model: bound by memory
        dict(name="append_prompts_70b", op="append", q_heads=64, kv_heads=8, head_dim=128, rotary=128, pairs="halves",
             fused_qkv=True, batch=16, prefix=700, spread=1.0, new=1900, lengths_seed=5),
        # the turn that eight chats just ended, on its way to the host tier, from 8-bit pools
        dict(name="read_turn_fp8", op="read", pools="fp8", q_heads=32, kv_heads=8, head_dim=128, batch=8, prefix=2560,
             spread=0.5, new=288, lengths_seed=3),
        # whole contexts that leave the 4-bit pools
        dict(name="read_contexts", op="read", pools="fp4", q_heads=64, kv_heads=8, head_dim=128, batch=12, prefix=0,
             spread=0.0, new=5500, lengths_seed=6),
        # three short answers of a tiny model: launches decide
        dict(name="attend_small", op="attend", entry="step", q_heads=4, kv_heads=1, head_dim=64, batch=3, prefix=170,
             spread=0.5, new=1, lengths_seed=7),
        # decoding of 32 conversations of the 70B model: bound by memory
        dict(name="attend_decode_70b", op="attend", entry="layer", q_heads=64, kv_heads=8, head_dim=128, batch=32,
             prefix=6500, spread=0.5, new=1, lengths_seed=8),
        # questions of about 20 tokens on cached contexts, d = 64
        dict(name="attend_questions_d64", op="attend", entry="step", q_heads=32, kv_heads=8, head_dim=64, batch=24,
             prefix=3000, spread=0.4, new=20, lengths_seed=10),
        # chat turns of the 8B model
        dict(name="attend_chat_8b", op="attend", entry="layer", q_heads=32, kv_heads=8, head_dim=128, batch=8, prefix=2560,
             spread=0.5, new=288, lengths_seed=3),
        # one user far into a long context: the whole step of a token
        dict(name="step_long_context", op="step", entry="step", q_heads=64, kv_heads=8, head_dim=128, rotary=128,
             pairs="halves", fused_qkv=True, batch=1, prefix=120011, spread=0.0, new=1, lengths_seed=11),
        # largest: prompts of about 800 tokens behind long contexts, 70B heads
        dict(name="attend_prompts_70b", op="attend", entry="layer", q_heads=64, kv_heads=8, head_dim=128, batch=6,
             prefix=9000, spread=0.3, new=800, lengths_seed=12),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads = rng.choice([(64, 8, 128), (64, 8, 128), (32, 8, 128), (8, 1, 128), (32, 8, 64), (16, 2, 128), (8, 8, 64)])
    c = dict(op=rng.choice(["append", "append", "read", "read", "attend", "attend", "attend", "step"]), q_heads=heads[0],
             kv_heads=heads[1], head_dim=heads[2], spread=0.6, lengths_seed=rng.randrange(1 << 30))
    if c["op"] in ("append", "step"):
        c.update(rotary=rng.choice([heads[2], heads[2], heads[2] // 2, 48, 0 if c["op"] == "append" else heads[2]]),
                 pairs=rng.choice(["halves", "interleaved"]))
        c.update(fused_qkv=c["rotary"] > 0 and rng.random() < 0.5)
    if c["op"] == "read":
        c.update(pools=rng.choice(["fp4", "fp4", "fp8", "bf16"]))
    if c["op"] in ("append", "read"):
        if rng.random() < 0.4:
            c.update(batch=_log_uniform(rng, 1, 256), prefix=_log_uniform(rng, 16, 8000), new=rng.choice([1, 1, 2, 5]))
        else:
            c.update(batch=_log_uniform(rng, 1, 32), prefix=rng.choice([0, _log_uniform(rng, 16, 4000)]),
                     new=_log_uniform(rng, 20, 5000))
    else:
        c.update(entry=rng.choice(["step", "layer"]))
        if rng.random() < 0.6:
            c.update(batch=_log_uniform(rng, 1, 128), prefix=_log_uniform(rng, 16, 60000), new=rng.choice([1, 1, 1, 2, 3]))
        else:
            c.update(batch=_log_uniform(rng, 1, 32), prefix=rng.choice([0, _log_uniform(rng, 16, 12000)]),
                     new=_log_uniform(rng, 4, 1500))
    most = {}
    for x in listed():
        most = {k: max(v, most.get(k, 0)) for k, v in work(x).items()}

    def too_much():
        P, n = lengths(c)
        L = int((P + n).max())
        return (any(work(c)[k] > most[k] for k in most) or
                (c["op"] in ("attend", "step") and (c["batch"] * c["q_heads"] * int(n.max()) * L > 4e9 or    # the plain form's
                                                    c["batch"] * c["kv_heads"] * c["head_dim"] * L > 1.5e9)))  # padded scores, keys
    while too_much():
        if c["batch"] > 1:
            c["batch"] = max(1, c["batch"] * 2 // 3)
        else:
            c["new"], c["prefix"] = max(1, c["new"] * 2 // 3), c["prefix"] * 2 // 3
    return c


def lengths(case):
    """(cached tokens, new tokens) of every request."""
    rng = np.random.default_rng(case["lengths_seed"])
    B = case["batch"]
    new = np.full(B, case["new"], np.int64)
    if case["new"] > 4:
        new = np.maximum(1, np.rint(case["new"] * rng.uniform(0.3, 1.7, B))).astype(np.int64)
    spread = np.exp(case["spread"] * rng.standard_normal(B)).clip(0.05, 4.0)
    return np.minimum(np.rint(case["prefix"] * spread).astype(np.int64), 131000), new


def _elem_bytes(case):
    """Bytes that an element takes in the pools, its share of the scales among them."""
    return {"fp4": 0.5 + 1 / 32, "fp8": 1, "bf16": 2}[case.get("pools", "fp4")]


def work(case):
    P, n = lengths(case)
    Hq, Hkv, D = case["q_heads"], case["kv_heads"], case["head_dim"]
    T = int(n.sum())
    total = dict(bytes=0.0, flops=0.0)
    if case["op"] in ("append", "step"):
        total["bytes"] += 2 * T * Hkv * D * (2 + _elem_bytes(case))
        total["flops"] += 2.0 * 2 * T * Hkv * D
        if case["rotary"]:
            positions = np.unique(np.concatenate([np.arange(p, p + m) for p, m in zip(P, n)])).size
            total["bytes"] += 2 * 2 * T * Hq * D + positions * case["rotary"] * 4
            total["flops"] += 3.0 * T * (Hq + Hkv) * case["rotary"]
    if case["op"] == "read":
        total["bytes"] += 2 * T * Hkv * D * (2 + _elem_bytes(case))
        total["flops"] += 2.0 * T * Hkv * D
    if case["op"] in ("attend", "step"):
        total["bytes"] += 2 * Hkv * D * _elem_bytes(case) * float((P + n).sum()) + 2 * 2 * Hq * D * T
        total["flops"] += 4.0 * D * Hq * float(np.sum(n * P + n * (n + 1) / 2))
    return total


# ------------------------------------------------------------------------------- inputs

def _table(positions, rotary):
    """(cos, sin) of every position and pair, angles in 64 bits."""
    inv = BASE ** (-torch.arange(0, rotary, 2, device="cuda", dtype=torch.float64) / rotary)
    angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * inv
    return torch.stack([angle.cos(), angle.sin()], dim=-1).float()


def _inputs(case, seed):
    """Keys with a few channels several times the others (as rotary models have them), values of unit variance,
    query heads at temperatures from 0.5 to 3 (nearly uniform to sharp attention). The pool is full (stale and
    other requests' tokens around this batch's), its pages in random order."""
    P, n = lengths(case)
    Hq, Hkv, D, B, T = case["q_heads"], case["kv_heads"], case["head_dim"], case["batch"], int(n.sum())
    rng = np.random.default_rng(seed)
    pages = -(-(P + n) // PAGE)
    # (an append or a read does not touch older pages: one block stands for all of them)
    first = P // PAGE if case["op"] in ("append", "read") else np.zeros(B, np.int64)
    used = int((pages - first).sum()) + 1
    order = rng.permutation(used + used // 8 + 2).astype(np.int32)
    tables = np.full((B, int(pages.max()) + 1), order[0], np.int32)
    at = 1
    for r in range(B):
        k = int(pages[r] - first[r])
        tables[r, first[r]:pages[r]] = order[at:at + k]
        at += k
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    channel = torch.ones(D, device="cuda", dtype=torch.bfloat16)
    channel[torch.from_numpy(rng.permutation(D)[:4]).cuda()] = 4.0
    heat = (0.5 * 6.0 ** (torch.arange(Hq, device="cuda") / max(1, Hq - 1))).to(torch.bfloat16)[None, :, None] / channel
    x = dict(P=P, n=n, tables=tables, scale=1.0 / math.sqrt(D))
    if case.get("fused_qkv"):   # views of the projection's one output
        qkv = normal(T, Hq + 2 * Hkv, D)
        qkv[:, :Hq] *= heat
        qkv[:, Hq:Hq + Hkv] *= channel
        x.update(q=qkv[:, :Hq], k_new=qkv[:, Hq:Hq + Hkv], v_new=qkv[:, Hq + Hkv:])
    else:
        x.update(q=normal(T, Hq, D) * heat)
        if case["op"] in ("append", "step"):
            x.update(k_new=normal(T, Hkv, D) * channel, v_new=normal(T, Hkv, D))
    k_pool, v_pool = normal(order.size, Hkv, PAGE, D) * channel, normal(order.size, Hkv, PAGE, D)
    kind = case.get("pools", "fp4")
    if kind == "fp4":
        (k_pool, ks), (v_pool, vs) = _quantise(k_pool.float()), _quantise(v_pool.float())
        x.update(scales=torch.stack([ks, vs], dim=-1))
    else:   # value pages of these pools are transposed
        v_pool = v_pool.transpose(2, 3).contiguous()
        if kind == "fp8":
            k_pool, v_pool = ((t.float() / s).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
                              for t, s in ((k_pool, 4 * K_SCALE), (v_pool, V_SCALE)))
    x.update(k_pool=k_pool, v_pool=v_pool)
    if case.get("rotary"):
        x["table"] = _table(-(-int((P + n).max()) // 1024) * 1024, case["rotary"])
    return x


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    P, n, T = s["P"], s["n"], int(s["n"].sum())
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int64)).cuda()  # noqa: E731
    row = np.repeat(np.arange(case["batch"]), n)                                  # request of each new token
    index = np.arange(T) - np.repeat(np.cumsum(n) - n, n)                         # and its place in it
    pos = P[row] + index
    s.update(pos=put(pos), row=put(row), index=put(index), block=put(s["tables"][row, pos // PAGE]), slot=put(pos % PAGE),
             prefix=put(P), new=put(n), cu=put(np.cumsum(n) - n), pages=put(s["tables"][:, :-(-int((P + n).max()) // PAGE)]),
             width=int(n.max()))
    rows = lambda heads: torch.empty(T, heads, case["head_dim"], dtype=torch.bfloat16, device="cuda")  # noqa: E731
    s.update(out=rows(case["q_heads"]), q_out=rows(case["q_heads"]), k_out=rows(case["kv_heads"]), v_out=rows(case["kv_heads"]))
    if own:   # the handle that a serving program makes once a batch, and the plan that its layers share
        import paper_2505_23970_amd as gc
        s["batch"] = gc.PagedBatch(P, n, s["tables"], device="cuda")
        if case["op"] in ("attend", "step"):
            s["workspace"] = gc.alloc_workspace(case["q_heads"], s["k_pool"], s["v_pool"], s["batch"])
            if case["entry"] == "layer":
                gc.plan(case["q_heads"], s["k_pool"], s["v_pool"], s["batch"], s["workspace"])
    return s


# ------------------------------------------------------------------------------- the calls

def _own_append(s):
    import paper_2505_23970_amd as gc
    c = s["case"]
    if not c["rotary"]:
        gc.kv_append_fp4(s["k_new"], s["v_new"], s["k_pool"], s["v_pool"], s["scales"], s["batch"])
        return None
    return gc.kv_append_rotary_fp4(s["q"], s["k_new"], s["v_new"], s["k_pool"], s["v_pool"], s["scales"], s["batch"],
                                   s["table"], q_out=s["q_out"], interleaved=c["pairs"] == "interleaved")


def _own_read(s):
    import paper_2505_23970_amd as gc
    pools, out = (s["k_pool"], s["v_pool"]), dict(k_out=s["k_out"], v_out=s["v_out"])
    kind = s["case"]["pools"]
    if kind == "fp4":
        return gc.kv_read_fp4(*pools, s["scales"], s["batch"], **out)
    if kind == "fp8":
        return gc.kv_read_fp8(*pools, s["batch"], 4 * K_SCALE, V_SCALE, **out)
    return gc.kv_read(*pools, s["batch"], **out)


def _own_attend(s, q):
    import paper_2505_23970_amd as gc
    call = gc.run_fp4 if s["case"]["entry"] == "layer" else gc.prefix_prefill_attention_fp4
    return call(q, s["k_pool"], s["v_pool"], s["scales"], s["batch"], s["scale"], s["workspace"], out=s["out"])


def run(s):
    op, got, q = s["case"]["op"], {}, s["q"]
    if op in ("append", "step"):
        turned = _own_append(s) if own else _append(s)
        if turned is not None:
            q = got["q"] = turned
        # the pools as they are: two codes a byte, whole numbers; the scales as the powers of two that they are
        got.update(k_codes=s["k_pool"], v_codes=s["v_pool"], scales=s["scales"].view(torch.float8_e8m0fnu))
    if op == "read":
        got["k"], got["v"] = _own_read(s) if own else _read(s)
    if op in ("attend", "step"):
        got["out"] = _own_attend(s, q) if own else _attend(s, q)
    return got


# ------------------------------------------------------------------------------- plain forms

def _quantise(x):
    """x float32 [..., D] as (codes uint8 [..., D/2], element 2i in the low half of byte i; scale codes uint8
    [..., D/32], 127 + e)."""
    b = x.unflatten(-1, (-1, 32))
    top = b.abs().amax(dim=-1)
    part, power = torch.frexp(top)                       # top = part 2^power, part in [0.5, 1)
    code = (power + 124 + (part >= 0.875)).clamp(3, 252)
    code = torch.where(top == 0, 3, code)
    a = b * torch.ldexp(torch.ones_like(top), 127 - code)[..., None]
    m = a.abs()
    e2m1 = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5)
            + 8 * torch.signbit(a).to(torch.uint8))
    e2m1 = e2m1.flatten(-2)
    return e2m1[..., 0::2] | e2m1[..., 1::2] << 4, code.to(torch.uint8)


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _values(codes, scale_codes):
    """The float32 numbers that codes [..., D/2] and scale codes [..., D/32] stand for."""
    e2m1 = torch.tensor(_E2M1, device="cuda")
    v = torch.stack([e2m1[(codes & 15).int()], e2m1[(codes >> 4).int()]], dim=-1).flatten(-2)
    s = scale_codes.contiguous().view(torch.float8_e8m0fnu).float()
    return (v.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def _rotate(x, cs, interleaved):
    """x [T][H][D], cs [T][R/2][2], both of one type."""
    half = cs.shape[1]
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        y[..., :half], y[..., half:2 * half] = a * cos - b * sin, b * cos + a * sin
    return y


def _append(s):
    k, v, interleaved = s["k_new"].float(), s["v_new"].float(), s["case"]["pairs"] == "interleaved"
    if s["case"]["rotary"]:
        cs = s["table"][s["pos"]]
        # (64 bits: a key next to the border of two codes has to fall on its own side)
        k = _rotate(s["k_new"].double(), cs.double(), interleaved).float()
        s["q_out"].copy_(_rotate(s["q"].float(), cs, interleaved))
    (kc, ks), (vc, vs) = _quantise(k), _quantise(v)
    s["k_pool"][s["block"], :, s["slot"]] = kc
    s["v_pool"][s["block"], :, s["slot"]] = vc
    s["scales"][s["block"], :, s["slot"]] = torch.stack([ks, vs], dim=-1)
    return s["q_out"] if s["case"]["rotary"] else None


def _read(s):
    kind, at = s["case"]["pools"], (s["block"], slice(None), s["slot"])
    if kind == "fp4":
        sc = s["scales"][at]
        k, v = _values(s["k_pool"][at], sc[..., 0]), _values(s["v_pool"][at], sc[..., 1])
    else:
        k, v = s["k_pool"][at], s["v_pool"][s["block"], :, :, s["slot"]]
        if kind == "fp8":
            k = k.contiguous().view(torch.float8_e4m3fn).float() * (4 * K_SCALE)
            v = v.contiguous().view(torch.float8_e4m3fn).float() * V_SCALE
    return s["k_out"].copy_(k), s["v_out"].copy_(v)


def _attend(s, q):
    """Every request's keys gathered (a padded batch), scores, softmax and sums in float32."""
    c = s["case"]
    Hkv, D, g, W = c["kv_heads"], c["head_dim"], c["q_heads"] // c["kv_heads"], s["width"]
    B, L = s["pages"].shape[0], s["pages"].shape[1] * PAGE
    sc = s["scales"][s["pages"]]                                 # [B][pages][Hkv][16][D/32][2]
    k, v = (_values(s[pool][s["pages"]], sc[..., i]).permute(0, 2, 1, 3, 4).reshape(B, Hkv, L, D)
            for i, pool in enumerate(("k_pool", "v_pool")))
    i = torch.arange(W, device="cuda")
    rows = (s["cu"][:, None] + torch.minimum(i, s["new"][:, None] - 1)).reshape(-1)   # (a short request repeats its last token)
    qp = q[rows].float().reshape(B, W, Hkv, g, D).transpose(1, 2).reshape(B, Hkv, W * g, D)
    x = torch.matmul(qp, k.transpose(2, 3)) * s["scale"]
    last = torch.minimum(s["prefix"][:, None] + i, (s["prefix"] + s["new"])[:, None] - 1)
    hidden = torch.arange(L, device="cuda") > last.repeat_interleave(g, dim=1)[:, None, :, None]
    x.masked_fill_(hidden, -math.inf)
    x.sub_(x.amax(dim=-1, keepdim=True)).exp_()
    o = torch.matmul(x, v) / x.sum(dim=-1, keepdim=True)
    o = o.reshape(B, Hkv, W, g, D).transpose(1, 2).reshape(B, W, Hkv * g, D)
    s["out"].copy_(o[s["row"], s["index"]])
    return s["out"]


# ------------------------------------------------------------------------------- what is right

def _blocks_exact(x):
    """(codes one a byte, scales) of float64 blocks [..., 32]: by distance to the sixteen values."""
    top = x.abs().amax(dim=-1)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -140) / 3.5))      # 3.5 s <= top < 7 s
    e = torch.where(top >= 7 * torch.exp2(e), e + 1, torch.where(top < 3.5 * torch.exp2(e), e - 1, e)).clamp(-124, 125)
    y = (x / torch.exp2(e)[..., None]).abs()
    best, code = y.clone(), torch.zeros(y.shape, dtype=torch.uint8, device="cuda")   # (distance to 0, code 0)
    for c in range(1, 8):
        d = (y - _E2M1[c]).abs()
        nearer = (d < best) | ((d == best) & (c % 2 == 0))
        best, code = torch.where(nearer, d, best), torch.where(nearer, c, code)
    return torch.where(torch.signbit(x), code + 8, code).to(torch.uint8), torch.exp2(e)


def exact(case, seed):
    """The definitions in float64, request by request and head by head. The step's attention takes the operands that
    its append hands over, rotated queries rounded to the type that holds them."""
    x = _inputs(case, seed)
    P, n, tables = x["P"], x["n"], x["tables"]
    Hq, Hkv, D, op, kind = case["q_heads"], case["kv_heads"], case["head_dim"], case["op"], case.get("pools", "fp4")
    got, q, kp, vp = {}, x["q"], x["k_pool"], x["v_pool"]
    value = torch.tensor(_E2M1, dtype=torch.float64, device="cuda")
    if kind == "fp4":   # one code a byte, and the blocks' scales
        one = lambda codes: torch.stack([codes % 16, codes // 16], dim=-1).flatten(-2)  # noqa: E731
        kp, vp, powers = one(kp), one(vp), torch.exp2(x["scales"].double() - 127)

    def rows(page, slot, h=slice(None)):
        if kind != "fp4":
            as_float = (lambda t, z: t.contiguous().view(torch.float8_e4m3fn).double() * float(np.float32(z))) if kind == "fp8" else (
                lambda t, z: t.double())
            return as_float(kp[page, h, slot], 4 * K_SCALE), as_float(vp[page, h, :, slot], V_SCALE)
        return tuple(value[pool[page, h, slot].int()] * powers[page, h, slot][..., i].repeat_interleave(32, dim=-1)
                     for i, pool in enumerate((kp, vp)))

    requests, cu = [], 0
    for r in range(case["batch"]):
        pos = torch.arange(int(P[r]), int(P[r] + n[r]), device="cuda")
        requests.append((cu, pos, torch.from_numpy(tables[r].astype(np.int64)).cuda()))
        cu += len(pos)
    if op == "read":
        both = [rows(page[pos // PAGE], pos % PAGE) for _, pos, page in requests]
        return {"k": torch.cat([k for k, _ in both]), "v": torch.cat([v for _, v in both])}
    if op in ("append", "step"):
        R, qs = case["rotary"], torch.empty(q.shape, dtype=torch.float64, device="cuda")
        first = torch.arange(0, R, 2, device="cuda") if case["pairs"] == "interleaved" else torch.arange(R // 2, device="cuda")
        second = first + (1 if case["pairs"] == "interleaved" else R // 2)
        for cu, pos, page in requests:
            turned = []
            for t in (q[cu:cu + len(pos)].double(), x["k_new"][cu:cu + len(pos)].double()):
                y = t.clone()
                if R:
                    cs = x["table"][pos].double()[:, None]
                    y[..., first] = t[..., first] * cs[..., 0] - t[..., second] * cs[..., 1]
                    y[..., second] = t[..., second] * cs[..., 0] + t[..., first] * cs[..., 1]
                turned.append(y)
            qs[cu:cu + len(pos)] = turned[0]
            at = (page[pos // PAGE], slice(None), pos % PAGE)
            for i, (pool, t) in enumerate(((kp, turned[1].float().double()), (vp, x["v_new"][cu:cu + len(pos)].double()))):
                codes, s = _blocks_exact(t.unflatten(-1, (-1, 32)))
                pool[at] = codes.flatten(-2)
                powers[at + (slice(None), i)] = s
        got = {"k_codes": kp[..., 0::2] + 16 * kp[..., 1::2], "v_codes": vp[..., 0::2] + 16 * vp[..., 1::2], "scales": powers}
        if R:
            got["q"], q = qs, qs.to(torch.bfloat16)
        if op == "append":
            return got
    g = Hq // Hkv
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    for cu, pos, page in requests:
        m, L = len(pos), int(pos[-1]) + 1
        j = torch.arange(L, device="cuda")
        seen = j[None, :] <= pos.repeat_interleave(g)[:, None]
        for h in range(Hkv):
            k, v = rows(page[j // PAGE], j % PAGE, h)
            z = torch.mm(q[cu:cu + m, h * g:(h + 1) * g].double().reshape(-1, D), k.t()) / math.sqrt(D)
            z = torch.where(seen, z, torch.full_like(z, -math.inf))
            out[cu:cu + m, h * g:(h + 1) * g] = torch.mm(torch.softmax(z, dim=1), v).reshape(m, g, D)
    return {**got, "out": out}
