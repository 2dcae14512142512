"""The operators around an 8-bit paged KV cache, as cases to be timed.

A decode step over a quantised cache rotates the new tokens' queries and keys,
quantises and stores their keys and values, and attends over the cache; a
finished sequence's rows are read back.  Four operations (`op`):

  rotary   rotary positions of query and key rows
  append   the new tokens' rows rotated, quantised and stored (queries rotated beside)
  decode   attention of `n` new tokens per sequence over the quantised cache
  read     a window of every sequence's keys and values back as bf16 rows

The cache.  A block holds 16 tokens.  A row of D values of one token and KV
head is stored as e4m3 codes times 2^(s - 127), s one byte: the smallest s >= 1
with max|x| <= 448 * 2^(s - 127), 0 for a row of zeros.

  k      e4m3 [blocks][Hkv][D/64][4][16][2][8], element d of slot o at [d/64][d/8%4][o][d/32%2][d%8]
  v      e4m3 [blocks][Hkv][2][4][D/8][2][8],   element d of slot o at [o/2%2][o/4][d/8][o%2][d%8]
  scale  uint8 [blocks][Hkv][2][16]: the bytes of the keys, then of the values

Sizes are those of the configurations in `workloads` and of the benchmark, or
generic ones in between.  Lengths are evenly spread quantiles of a case's
distribution (so that a case costs the same whatever the seed) in an order
drawn from the seed; blocks are scattered over the pool.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16


def listed():
    return [
        # One decode step's queries and keys: small, a launch is most of it.
        dict(name="rotary_step", op="rotary", tokens=256, q_heads=32, kv_heads=8, head_dim=128, rotary_dim=128,
             interleaved=False, backward=False, dtype="bf16", base=500000.0, longest=4096),
        # The gradient of a packed training batch's rotated rows, neighbouring pairs, half of every head.
        dict(name="rotary_train", op="rotary", tokens=16384, q_heads=28, kv_heads=4, head_dim=128, rotary_dim=64,
             interleaved=True, backward=True, dtype="bf16", base=1000000.0, longest=8192),
        # One new token of every running sequence, its query rotated in the same call.
        dict(name="append_step", op="append", batch=256, q_heads=32, kv_heads=8, head_dim=128, n=1, rotary_dim=128,
             interleaved=False, base=500000.0, dist="uniform", lo=1, hi=64),
        # New prompts of up to 1024 tokens, aligned to their ends (a shorter prompt's first rows are padding).
        dict(name="append_prompts", op="append", batch=48, q_heads=28, kv_heads=4, head_dim=128, n=1024,
             rotary_dim=128, interleaved=False, base=1000000.0, dist="uniform", lo=64, hi=1024),
        # The smallest step: a handful of short sequences, where the call itself is the cost.
        dict(name="decode_tiny", op="decode", batch=4, q_heads=8, kv_heads=2, head_dim=64, n=1,
             dist="uniform", lo=1, hi=257),
        # The end of a rollout: a few long samples are left in the batch.
        dict(name="decode_few_long", op="decode", batch=8, q_heads=32, kv_heads=8, head_dim=128, n=1,
             dist="loguniform", lo=512, hi=16384),
        # The headline decode step (Llama-3-8B shape).
        dict(name="decode_8b", op="decode", batch=256, q_heads=32, kv_heads=8, head_dim=128, n=1,
             dist="uniform", lo=512, hi=4096),
        # One GPU's share of a TP=8 Llama-3-70B layer: one KV head, split contexts.
        dict(name="decode_70b_tp8", op="decode", batch=512, q_heads=8, kv_heads=1, head_dim=128, n=1,
             dist="uniform", lo=1024, hi=8192),
        # Verification of four drafted tokens and the one after them.
        dict(name="verify_8b", op="decode", batch=256, q_heads=32, kv_heads=8, head_dim=128, n=5,
             dist="uniform", lo=512, hi=4096),
        # Chunked prefill: 512 tokens of each prompt over what is cached.
        dict(name="chunked_prefill", op="decode", batch=32, q_heads=32, kv_heads=8, head_dim=128, n=512,
             dist="uniform", lo=1024, hi=8192),
        # A few rows of a few sequences, odd windows (what a recomputation of the last tokens starts from).
        dict(name="read_window", op="read", batch=5, kv_heads=2, head_dim=64, dist="uniform", lo=70, hi=333,
             window=61),
        # Whole finished rollouts handed over.
        dict(name="read_rollouts", op="read", batch=64, kv_heads=8, head_dim=128, dist="uniform", lo=512, hi=4096,
             window=0),
    ]


HEADS = [(8, 2, 64), (32, 8, 128), (8, 1, 128), (28, 4, 128), (40, 8, 128), (12, 2, 128), (16, 16, 64), (16, 1, 128)]
MOST_BYTES, MOST_FLOPS = 1.2e9, 1.1e12
MOST_SCORES = 5.0e9  # scores that the plain form holds at once


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes spread over the logarithm of their ranges, no more
    work than the largest listed."""
    op = rng.choice(["decode"] * 6 + ["append"] * 2 + ["rotary"] * 2 + ["read"] * 2)
    hq, hkv, d = rng.choice(HEADS)
    case = dict(op=op, kv_heads=hkv, head_dim=d)
    if op != "read":
        case["q_heads"] = hq
    if op in ("rotary", "append"):
        case["rotary_dim"] = 16 * rng.randint(1, d // 16)
        case["interleaved"] = rng.random() < 0.5
        case["base"] = rng.choice([1e4, 5e5, 1e6])
    if op == "rotary":
        case.update(tokens=_log(rng, 1, 20000), backward=rng.random() < 0.3, dtype=rng.choice(["bf16", "bf16", "f32"]),
                    longest=_log(rng, 16, 100000))
        while _too_much(case):
            case["tokens"] = case["tokens"] * 2 // 3
        return case
    case["dist"] = rng.choice(["uniform", "loguniform"])
    hi = _log(rng, 16, 16384 if op == "decode" else 4096)
    if op in ("decode", "append"):
        case["n"] = _log(rng, 1, 1024) if rng.random() < 0.6 else 1
        hi = max(hi, case["n"])
    case["lo"], case["hi"] = max(1, min(hi, _log(rng, max(1, hi // 32), hi))), hi
    case["batch"] = _log(rng, 1, 512)
    if op == "read":
        case["window"] = 0 if rng.random() < 0.5 else _log(rng, 1, hi)
    while case["batch"] > 1 and _too_much(case):
        case["batch"] = case["batch"] * 2 // 3
    while _too_much(case):
        case["hi"] = case["hi"] * 2 // 3
        case["lo"] = min(case["lo"], case["hi"])
        if "n" in case:
            case["n"] = min(case["n"], case["hi"])
    return case


def _too_much(case):
    w = work(case)
    if w["bytes"] > MOST_BYTES or w["flops"] > MOST_FLOPS:
        return True
    if case["op"] == "rotary":
        return False
    padded = case["batch"] * -(-case["hi"] // BLOCK) * BLOCK
    if case["op"] == "decode" and padded * case["q_heads"] * case["n"] > MOST_SCORES:
        return True
    return padded * case["kv_heads"] * case["head_dim"] > 1.2e9


# ------------------------------------------------------------------ sizes --

def _lens(case, seed=None):
    """Context lengths: evenly spread quantiles of the case's distribution, shuffled by the seed."""
    u = (np.arange(case["batch"]) + 0.5) / case["batch"]
    lo, hi = case["lo"], case["hi"]
    x = lo + u * (hi - lo) if case["dist"] == "uniform" else lo * (hi / lo) ** u
    x = np.clip(np.rint(x), lo, hi).astype(np.int64)
    return x if seed is None else np.random.RandomState(seed % (1 << 31)).permutation(x)


def _window(case, lens):
    """First token and token count that a read takes of every sequence: all of it, or the last `window`."""
    count = np.minimum(lens, case["window"]) if case["window"] else lens
    return lens - count, count


def work(case):
    hkv, d = case["kv_heads"], case["head_dim"]
    if case["op"] == "rotary":
        T, size = case["tokens"], 2 if case["dtype"] == "bf16" else 4
        rows = (T - T // 50) * (case["q_heads"] + hkv)
        return dict(bytes=float(2 * rows * d * size + 4 * T), flops=float(3 * rows * case["rotary_dim"]))
    lens = _lens(case)
    B = len(lens)
    if case["op"] == "read":
        rows = int(_window(case, lens)[1].sum())
        return dict(bytes=float(rows * hkv * (2 * d + 2 + 4 * d) + 4 * -(-rows // BLOCK)), flops=float(2 * rows * hkv * d))
    n, hq = case["n"], case["q_heads"]
    new = int(np.minimum(lens, n).sum())
    if case["op"] == "append":
        return dict(bytes=float(new * (4 * hq * d + 2 * hkv * (2 * d + d + 1)) + 4 * -(-new // BLOCK) + 4 * B),
                    flops=float(new * (hq + 2 * hkv) * 3 * d))
    visible = sum(int(np.clip(lens - n + 1 + i, 0, None).sum()) for i in range(n))
    return dict(bytes=float(lens.sum() * hkv * (2 * d + 2) + 6 * new * hq * d + 4 * (-(-lens // BLOCK)).sum() + 4 * B),
                flops=float(4 * d * hq * visible))


# ----------------------------------------------------------------- inputs --

def _quantised(x):
    """Codes (e4m3) and scale bytes of rows x [..., D] in fp32."""
    m, e = torch.frexp(x.abs().amax(-1))  # amax = m 2^e, m in [0.5, 1)
    s = (torch.where(m <= 0.875, e - 9, e - 8) + 127).clamp(min=1)  # 448 = 0.875 * 2^9
    codes = (x * ((254 - s) << 23).view(torch.float32)[..., None]).to(torch.float8_e4m3fn)  # x 2^(127 - s), exactly
    return codes, torch.where(m > 0, s, 0).to(torch.uint8)


def _pool(case, seed, filled):
    """Block table, lengths and cache of a case's sequences on the GPU."""
    dev = torch.device("cuda")
    hkv, d = case["kv_heads"], case["head_dim"]
    lens = _lens(case, seed)
    blocks = -(-lens // BLOCK)
    NB, width = int(math.ceil(1.1 * blocks.sum())), int(blocks.max())
    perm = np.random.RandomState((seed + 1) % (1 << 31)).permutation(NB).astype(np.int32)
    table, used = np.full((len(lens), width), -1, np.int32), 0
    for b, m in enumerate(blocks):
        table[b, :m] = perm[used:used + m]
        used += int(m)
    f8 = torch.float8_e4m3fn
    k = torch.zeros((NB, hkv, d // 64, 4, BLOCK, 2, 8), dtype=torch.uint8, device=dev).view(f8)
    v = torch.zeros((NB, hkv, 2, 4, d // 8, 2, 8), dtype=torch.uint8, device=dev).view(f8)
    scale = torch.zeros((NB, hkv, 2, BLOCK), dtype=torch.uint8, device=dev)
    if filled:
        gen = torch.Generator(device=dev)
        gen.manual_seed(seed)
        # Keys carry an offset per head and channel and a few strong channels, values differ in size from
        # token to token, as trained attention has.
        offset = torch.randn((hkv, 1, d), generator=gen, device=dev) * 0.5
        offset[:, :, ::37] *= 6
        kc, scale[:, :, 0] = _quantised(torch.randn((NB, hkv, BLOCK, d), generator=gen, device=dev) + offset)
        k.view(torch.uint8).copy_(kc.view(torch.uint8).view(NB, hkv, BLOCK, d // 64, 2, 4, 8).permute(0, 1, 3, 5, 2, 4, 6))
        size = torch.exp2(torch.randn((NB, hkv, BLOCK, 1), generator=gen, device=dev))
        vc, scale[:, :, 1] = _quantised(torch.randn((NB, hkv, BLOCK, d), generator=gen, device=dev) * size)
        v.view(torch.uint8).copy_(vc.view(torch.uint8).view(NB, hkv, 4, 2, 2, d // 8, 8).permute(0, 1, 3, 2, 5, 4, 6))
    return dict(k=k, v=v, scale=scale, table=torch.from_numpy(table).to(dev),
                lens=torch.from_numpy(lens.astype(np.int32)).to(dev), host_lens=lens, longest=int(lens.max()))


def _inv_freq(case):
    i = np.arange(case["rotary_dim"] // 2)
    return torch.from_numpy(case["base"] ** (-2.0 * i / case["rotary_dim"])).cuda()


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed + 7)
    hkv, d = case["kv_heads"], case["head_dim"]
    state = dict(case)
    if case["op"] == "rotary":
        # a packed batch: sequences of up to `longest` tokens one after the other, padded to its size at the end
        T, rng, pos = case["tokens"], np.random.RandomState(seed % (1 << 31)), []
        while len(pos) < T:
            start = rng.randint(case["longest"])
            pos += list(range(start, case["longest"]))[:rng.randint(1, 1 + min(T, case["longest"]))]
        pos = np.array(pos[:T], np.int32)
        pos[T - T // 50:] = -1
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        # rows of the fused projection: a token's queries, keys and values side by side
        rows = torch.randn((T, case["q_heads"] + 2 * hkv, d), generator=gen, device=dev).to(dtype)
        state.update(q=rows[:, :case["q_heads"]], k=rows[:, case["q_heads"]:case["q_heads"] + hkv],
                     positions=torch.from_numpy(pos).to(dev), inv_freq=_inv_freq(case))
        state["q_out"] = torch.zeros((T, case["q_heads"], d), dtype=dtype, device=dev)
        state["k_out"] = torch.zeros((T, hkv, d), dtype=dtype, device=dev)
        return state
    state.update(_pool(case, seed, case["op"] != "append"))
    lens, B = state["host_lens"], case["batch"]
    if case["op"] == "read":
        first, count = _window(case, lens)
        start = np.concatenate([[0], np.cumsum(count)])
        state["first"] = torch.from_numpy(first.astype(np.int32)).to(dev)
        state["row_start"] = torch.from_numpy(start.astype(np.int32)).to(dev)
        seq = np.repeat(np.arange(B), count)
        at = np.arange(start[-1]) - start[seq] + first[seq]
        state["seq"], state["at"] = torch.from_numpy(seq).to(dev), torch.from_numpy(at).to(dev)
        state["k_out"] = torch.zeros((int(start[-1]), hkv, d), dtype=torch.bfloat16, device=dev)
        state["v_out"] = torch.zeros_like(state["k_out"])
        return state
    n, hq = case["n"], case["q_heads"]
    state["q"] = (torch.randn((B, n, hq, d), generator=gen, device=dev) * 1.5).to(torch.bfloat16)
    if case["op"] == "decode":
        state["softmax_scale"] = 1.0 / math.sqrt(d)
        state["out"] = torch.zeros((B, n, hq, d), dtype=torch.float32, device=dev)
        return state
    offset = torch.randn((hkv, d), generator=gen, device=dev) * 0.5
    offset[:, ::37] *= 6
    state["k_new"] = (torch.randn((B, n, hkv, d), generator=gen, device=dev) + offset).to(torch.bfloat16)
    state["v_new"] = torch.randn((B, n, hkv, d), generator=gen, device=dev).to(torch.bfloat16)
    state["q_out"] = torch.zeros_like(state["q"])
    state["inv_freq"] = _inv_freq(case)
    # the rows that are no padding, and their places in the contexts
    seq = np.repeat(np.arange(B), np.minimum(lens, n))
    at = np.concatenate([np.arange(max(0, x - n), x) for x in lens])
    state["seq"], state["at"] = torch.from_numpy(seq).to(dev), torch.from_numpy(at).to(dev)
    state["row"] = torch.from_numpy(at - lens[seq] + n).to(dev)
    return state


# -------------------------------------------------------------------- run --

def run(state):
    if own:
        return _own(state)
    return {"rotary": _rotary, "append": _append, "decode": _decode, "read": _read}[state["op"]](state)


def _own(state):
    """The framework's call, its arguments bound on a state's first pass as a serving loop binds them."""
    import paper_2405_11143_amd as pda

    op = state["op"]
    if "call" not in state:
        if op in ("rotary", "append"):
            rotary = pda.make_rotary(state["inv_freq"], interleaved=state["interleaved"],
                                     backward=state.get("backward", False))
        if op == "rotary":
            state["call"] = pda.bind_rotary_apply(state["q"], state["positions"], rotary, k=state["k"],
                                                  q_out=state["q_out"], k_out=state["k_out"])
        else:
            cache = (state["k"], state["v"], state["scale"])
            paged = (state["table"], state["lens"])
        if op == "append":
            state["call"] = pda.bind_append_kv_fp8(state["k_new"], state["v_new"], *paged, *cache, rotary=rotary,
                                                   q=state["q"], q_out=state["q_out"], max_context_len=state["longest"])
        elif op == "decode":
            state["call"] = pda.bind_decode_fp8(state["q"], *cache, *paged, state["softmax_scale"], state["out"],
                                                max_context_len=state["longest"])
        elif op == "read":
            state["call"] = pda.bind_read_kv_fp8(*cache, *paged, state["row_start"], state["k_out"], state["v_out"],
                                                 first_token=state["first"], max_context_len=state["longest"])
    state["call"]()
    return _outputs(state)


def _outputs(state):
    if state["op"] == "rotary":
        return dict(q=state["q_out"], k=state["k_out"])
    if state["op"] == "append":  # the cache as the values that its codes and bytes stand for
        return dict(q=state["q_out"], k=state["k"], v=state["v"], scale=state["scale"].view(torch.float8_e8m0fnu))
    if state["op"] == "decode":
        return dict(out=state["out"])
    return dict(k=state["k_out"], v=state["v_out"])


def _rotated(x, positions, state, backward=False):
    """fp32 rows x [T, H, D] at positions [T], rotated."""
    R = state["rotary_dim"]
    angle = positions.to(torch.float64)[:, None] * state["inv_freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if backward:
        sin = -sin
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if state["interleaved"] else (x[..., :R // 2], x[..., R // 2:R])
    c, e = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([c, e], -1).flatten(-2) if state["interleaved"] else torch.cat([c, e], -1)
    return torch.cat([turned, x[..., R:]], -1)


def _rotary(state):
    real = (state["positions"] >= 0)[:, None, None]
    for name in ("q", "k"):
        y = _rotated(state[name].float(), state["positions"], state, state["backward"]).to(state[name].dtype)
        state[name + "_out"].copy_(torch.where(real, y, state[name + "_out"]))
    return _outputs(state)


def _append(state):
    seq, at, row = state["seq"], state["at"], state["row"]
    d, hkv = state["head_dim"], state["kv_heads"]
    block, slot = state["table"][seq, at // BLOCK].long(), at % BLOCK
    state["q_out"][seq, row] = _rotated(state["q"][seq, row].float(), at, state).to(torch.bfloat16)
    k, ks = _quantised(_rotated(state["k_new"][seq, row].float(), at, state))
    v, vs = _quantised(state["v_new"][seq, row].float())
    k8, v8 = state["k"].view(torch.uint8), state["v"].view(torch.uint8)
    k8[block, :, :, :, slot] = k.view(torch.uint8).view(-1, hkv, d // 64, 2, 4, 8).transpose(3, 4)
    # (indices apart from each other: the indexed axis comes first)
    v8.permute(0, 3, 2, 5, 1, 4, 6)[block, slot // 4, slot // 2 % 2, slot % 2] = v.view(torch.uint8).view(-1, hkv, d // 8, 8)
    state["scale"][block, :, 0, slot] = ks
    state["scale"][block, :, 1, slot] = vs
    return _outputs(state)


def _factor(scale):
    return (scale.int() << 23).view(torch.float32)  # 2^(s - 127), 0 for 0


def _decode(state):
    B, n, hq, d = state["q"].shape
    hkv = state["kv_heads"]
    G, ids = hq // hkv, state["table"].clamp(min=0).long()
    T = ids.shape[1] * BLOCK
    scale = _factor(state["scale"][ids])  # [B, blocks, hkv, 2, 16]
    k = state["k"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).float()  # [B, blocks, hkv, d/64, 4, 16, 2, 8]
    k = k.permute(0, 2, 1, 5, 3, 6, 4, 7).reshape(B, hkv, T, d) * scale[:, :, :, 0].transpose(1, 2).reshape(B, hkv, T, 1)
    q = state["q"].float().view(B, n, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * G, d)
    s = torch.matmul(q, k.transpose(2, 3)) * state["softmax_scale"]
    del k
    token = torch.arange(T, device=s.device)
    limit = state["lens"][:, None] - n + 1 + torch.arange(n, device=s.device)  # [B, n]
    hidden = (token >= limit[:, :, None])[:, None, :, None]  # [B, 1, n, 1, T]
    s = s.view(B, hkv, n, G, T).masked_fill_(hidden, -math.inf).view(B, hkv, n * G, T)
    s = s.sub_(s.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = s.sum(-1, keepdim=True)
    v = state["v"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).float()  # [B, blocks, hkv, 2, 4, d/8, 2, 8]
    v = v.permute(0, 2, 1, 4, 3, 6, 5, 7).reshape(B, hkv, T, d) * scale[:, :, :, 1].transpose(1, 2).reshape(B, hkv, T, 1)
    out = torch.matmul(s, v) / total.clamp(min=1e-30)
    return dict(out=out.view(B, hkv, n, G, d).permute(0, 2, 1, 3, 4).reshape(B, n, hq, d))


def _read(state):
    seq, at = state["seq"], state["at"]
    d, hkv = state["head_dim"], state["kv_heads"]
    block, slot = state["table"][seq, at // BLOCK].long(), at % BLOCK
    scale = _factor(state["scale"].transpose(2, 3).transpose(1, 2)[block, slot])  # [rows, hkv, 2]
    k = state["k"].view(torch.uint8)[block, :, :, :, slot].view(torch.float8_e4m3fn).float()  # [rows, hkv, d/64, 4, 2, 8]
    v = state["v"].view(torch.uint8).permute(0, 3, 2, 5, 1, 4, 6)[block, slot // 4, slot // 2 % 2, slot % 2]
    state["k_out"].copy_(k.transpose(3, 4).reshape(-1, hkv, d) * scale[:, :, :1])
    state["v_out"].copy_(v.view(torch.float8_e4m3fn).float().reshape(-1, hkv, d) * scale[:, :, 1:])
    return _outputs(state)


# -------------------------------------------------------------- reference --

def _e4m3(y):
    """y (64 bits) rounded to the nearest e4m3 value, ties to even."""
    _, e = torch.frexp(y)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return torch.round(y / step) * step


def _exact_rotary(x, pos, inv_freq, case, sign):
    """Rows x [T, H, D] in 64 bits, each pair as a complex number turned by its angle."""
    R = case["rotary_dim"]
    turn = torch.polar(torch.ones((len(pos), R // 2), dtype=torch.float64, device=x.device), sign * pos.double()[:, None] * inv_freq)
    y = x.clone()
    first = slice(0, R, 2) if case["interleaved"] else slice(0, R // 2)
    second = slice(1, R, 2) if case["interleaved"] else slice(R // 2, R)
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn[:, None]
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    state = prepare(case, seed)
    f64, d, hkv = torch.float64, case["head_dim"], case["kv_heads"]
    if case["op"] == "rotary":
        out, real = {}, state["positions"] >= 0
        for name in ("q", "k"):
            y = _exact_rotary(state[name].to(f64), state["positions"], state["inv_freq"], case, -1 if case["backward"] else 1)
            out[name] = torch.where(real[:, None, None], y, 0.0)
        return out
    lens = state["host_lens"]
    d_of = torch.arange(d, device="cuda")
    o_of = torch.arange(BLOCK, device="cuda")[:, None]

    def rows_of(ids):
        """Keys and values [tokens, hkv, d] of the listed blocks, element by element from the layouts."""
        kb, vb = (state[x].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double() for x in ("k", "v"))
        kb = kb[:, :, d_of // 64, d_of // 8 % 4, o_of, d_of // 32 % 2, d_of % 8]
        vb = vb[:, :, o_of // 2 % 2, o_of // 4, d_of // 8, o_of % 2, d_of % 8]
        s = state["scale"][ids].double()
        s = torch.where(s > 0, torch.exp2(s - 127), 0.0)
        return [(x * s[:, :, i, :, None]).transpose(1, 2).reshape(-1, hkv, d) for i, x in enumerate((kb, vb))]

    if case["op"] == "read":
        first, count = _window(case, lens)
        got = []
        for b, x in enumerate(lens):
            kb, vb = rows_of(state["table"][b, :-(-x // BLOCK)].long())
            got.append((kb[first[b]:first[b] + count[b]], vb[first[b]:first[b] + count[b]]))
        return dict(k=torch.cat([g[0] for g in got]), v=torch.cat([g[1] for g in got]))
    B, n, hq = case["batch"], case["n"], case["q_heads"]
    if case["op"] == "append":
        out = dict(q=torch.zeros((B, n, hq, d), dtype=f64, device="cuda"), k=state["k"].double(), v=state["v"].double(),
                   scale=torch.full(state["scale"].shape, 2.0 ** -127, dtype=f64, device="cuda"))
        for b, x in enumerate(lens):
            t = torch.arange(max(0, x - n), x, device="cuda")
            i, page, slot = t - (x - n), state["table"][b, t // BLOCK].long(), (t % BLOCK)[:, None]
            out["q"][b, i] = _exact_rotary(state["q"][b, i].double(), t, state["inv_freq"], case, 1)
            for which, name in enumerate(("k", "v")):
                y = state[name + "_new"][b, i].double()
                if name == "k":
                    y = _exact_rotary(y, t, state["inv_freq"], case, 1)
                p = torch.ceil(torch.log2(y.abs().amax(-1) / 448))  # (no row here is zero, or anywhere near 2^-126)
                codes = _e4m3(y / torch.exp2(p)[..., None])
                if name == "k":
                    at = (page[:, None], slice(None), d_of // 64, d_of // 8 % 4, slot, d_of // 32 % 2, d_of % 8)
                else:
                    at = (page[:, None], slice(None), slot // 2 % 2, slot // 4, d_of // 8, slot % 2, d_of % 8)
                out[name][at] = codes.transpose(1, 2)
                out["scale"][page, :, which, slot[:, 0]] = torch.exp2(p)
        return out
    G = hq // hkv
    out = torch.zeros((B, n, hq, d), dtype=f64, device="cuda")
    for b, x in enumerate(lens):
        x = int(x)
        kb, vb = rows_of(state["table"][b, :-(-x // BLOCK)].long())
        i0 = max(0, n - x)
        seen = torch.arange(x - n + i0, x, device="cuda")[:, None, None]
        after = torch.arange(x, device="cuda") > seen  # [rows, 1, tokens]
        for g in range(hkv):
            qb = state["q"][b, i0:, g * G:(g + 1) * G].double()
            w = (qb.reshape(-1, d) @ kb[:x, g].T).view(n - i0, G, x) * case["head_dim"] ** -0.5
            w = torch.softmax(w.masked_fill(after, -math.inf), -1)
            out[b, i0:, g * G:(g + 1) * G] = (w.view(-1, x) @ vb[:x, g]).view(n - i0, G, d)
    return dict(out=out)
