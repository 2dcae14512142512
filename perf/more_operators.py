"""More operators of a model's step around the paged KV cache, as cases to be timed.

A layer that norms its query and key heads before their positions are applied, keys
stored through a slot map, attention that sees a sliding window and the first few
tokens, and the block tables and slot maps themselves, kept on the GPU (`op`):

  rotary   rotary positions with several axes (time, height, width), and their gradient
  norm     RMS norms of every query and key head and the rotation, in one pass; `backward`:
           the gradients of that pass with respect to the rows and the norms' weights
  store    the pass of `norm` with its keys, and the values, stored in the paged cache
  window   attention of `n` new tokens per sequence that see the last `window` tokens up
           to their own, and the first `sinks`
  blocks   a batch's block tables grown to new lengths, with the positions and slots of
           the new tokens, and shrunk again

The cache is the bf16 one: k [blocks][Hkv][D/8][16][8], v [blocks][Hkv][16][D].  A slot
is 16 * block + place in the block.

Block tables.  Every sequence's row holds the ids of the blocks of its first `held`
entries; free blocks are a stack.  Growing hands out ids from its top, in the order of
the sequences and of the entries in each; a sequence whose blocks are not all there
gets none, and none after it.  Shrinking puts ids back so that growing again hands out
the same ids.  Entries past `held` keep what they had.

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
        # Positions of a batch of prompts with images: text, then patches at (time, height, width).
        dict(name="rotary_images", op="rotary", tokens=6000, q_heads=28, kv_heads=4, head_dim=128, rotary_dim=128,
             interleaved=False, backward=False, dtype="bf16", base=1000000.0, axes=3),
        # The gradient of a vision encoder's rotated rows, in fp32: two axes, neighbouring pairs.
        dict(name="rotary_patches_grad", op="rotary", tokens=4097, q_heads=16, kv_heads=16, head_dim=64, rotary_dim=64,
             interleaved=True, backward=True, dtype="f32", base=10000.0, axes=2),
        # A packed training batch, forward and backward.
        dict(name="norm_train", op="norm", tokens=16384, q_heads=32, kv_heads=8, head_dim=128, rotary_dim=128,
             interleaved=False, backward=False, dtype="bf16", base=1000000.0, axes=1),
        dict(name="norm_train_grad", op="norm", tokens=16384, q_heads=32, kv_heads=8, head_dim=128, rotary_dim=128,
             interleaved=False, backward=True, dtype="bf16", base=1000000.0, axes=1),
        # A decode step's new tokens: queries for the attention, keys and values into the cache.
        dict(name="store_step", op="store", batch=256, q_heads=32, kv_heads=8, head_dim=128, rotary_dim=128, n=1,
             interleaved=False, base=1000000.0, axes=1, dist="uniform", lo=512, hi=4096),
        # New prompts one after the other without padding.
        dict(name="store_prompts", op="store", batch=48, q_heads=28, kv_heads=4, head_dim=128, rotary_dim=128, n=1024,
             interleaved=False, base=1000000.0, axes=1, dist="uniform", lo=64, hi=1024),
        # The smallest attention step: a handful of short sequences.
        dict(name="window_tiny", op="window", batch=4, q_heads=8, kv_heads=2, head_dim=64, n=1, window=64, sinks=4,
             dist="uniform", lo=1, hi=257),
        # A decode step of a whole rollout batch (Llama-3-8B shape), contexts mostly past the window.
        dict(name="window_8b", op="window", batch=256, q_heads=32, kv_heads=8, head_dim=128, n=1, window=1024, sinks=4,
             dist="uniform", lo=512, hi=4096),
        # The end of a rollout: a few long samples, a wide window.
        dict(name="window_few_long", op="window", batch=8, q_heads=32, kv_heads=8, head_dim=128, n=1, window=4096,
             sinks=16, dist="loguniform", lo=512, hi=16384),
        # Chunked prefill: 512 tokens of each prompt over what is cached.
        dict(name="window_chunk", op="window", batch=32, q_heads=32, kv_heads=8, head_dim=128, n=512, window=1024,
             sinks=4, dist="uniform", lo=1024, hi=8192),
        # Verification of four drafted tokens: blocks for them, and back where they are rejected.
        dict(name="blocks_verify", op="blocks", batch=256, n=5, kept=2, dist="uniform", lo=512, hi=4096),
        # A batch of prompts admitted and, later, all of it released.
        dict(name="blocks_prompts", op="blocks", batch=512, n=4096, kept=0, dist="uniform", lo=64, hi=4096),
    ]


HEADS = [(8, 2, 64), (32, 8, 128), (8, 1, 128), (28, 4, 128), (40, 8, 128), (12, 2, 128), (16, 16, 64), (16, 1, 128)]
OTHER_HEADS = [(16, 16, 80), (16, 4, 256)]  # of rows that meet no cache
MOST_BYTES, MOST_FLOPS = 9.0e8, 2.5e11
MOST_SCORES = 8.0e8  # scores, and elements of gathered rows, that the plain form holds at once


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes spread over the logarithm of their ranges, no more
    work than the largest listed."""
    op = rng.choice(["rotary", "norm", "norm", "store", "window", "window", "window", "blocks"])
    if op == "blocks":
        hi = _log(rng, 4, 8192)
        case = dict(op=op, batch=_log(rng, 1, 1024), n=_log(rng, 1, hi), dist=rng.choice(["uniform", "loguniform"]))
        case.update(kept=rng.randint(0, case["n"]), lo=max(1, min(hi, _log(rng, max(1, hi // 32), hi))), hi=hi)
        while case["batch"] > 1 and case["batch"] * case["hi"] > 2.5e6:
            case["batch"] = case["batch"] * 2 // 3
        return case
    hq, hkv, d = rng.choice(HEADS + OTHER_HEADS if op in ("rotary", "norm") else HEADS)
    case = dict(op=op, q_heads=hq, kv_heads=hkv, head_dim=d)
    if op != "window":
        case.update(rotary_dim=16 * rng.randint(1, d // 16), interleaved=rng.random() < 0.5,
                    base=rng.choice([1e4, 5e5, 1e6]), axes=rng.choice([1, 1, 2, 3, 3, 4]))
    if op in ("rotary", "norm"):
        case.update(tokens=_log(rng, 1, 20000), dtype=rng.choice(["bf16", "bf16", "f32"]), backward=rng.random() < 0.4)
        while _too_much(case):
            case["tokens"] = case["tokens"] * 2 // 3
        return case
    case["dist"] = rng.choice(["uniform", "loguniform"])
    hi = _log(rng, 16, 16384 if op == "window" else 4096)
    case["n"] = _log(rng, 1, 1024) if rng.random() < 0.6 else 1
    hi = max(hi, case["n"])
    case["lo"], case["hi"] = max(1, min(hi, _log(rng, max(1, hi // 32), hi))), hi
    case["batch"] = _log(rng, 1, 512)
    if op == "window":
        case.update(window=_log(rng, 1, 8192), sinks=rng.choice([0, 1, 4, 4, 16, 61, 128]))
    while case["batch"] > 1 and _too_much(case):
        case["batch"] = case["batch"] * 2 // 3
    while _too_much(case):
        case["hi"] = case["hi"] * 2 // 3
        case["lo"], case["n"] = min(case["lo"], case["hi"]), min(case["n"], case["hi"])
    return case


def _too_much(case):
    w = work(case)
    if w["bytes"] > MOST_BYTES or w["flops"] > MOST_FLOPS:
        return True
    if case["op"] not in ("window", "store"):
        return False
    if case["op"] == "window":
        seen = case["batch"] * min(case["hi"], case["sinks"] + case["window"] + case["n"])
        if seen * max(case["q_heads"] * case["n"], 2 * case["kv_heads"] * case["head_dim"]) > MOST_SCORES:
            return True
    return case["batch"] * case["hi"] * case["kv_heads"] * case["head_dim"] > 1.2e9


# ------------------------------------------------------------------ sizes --

def _lens(case, seed=None):
    """Lengths: evenly spread quantiles of the case's distribution, shuffled by the seed."""
    u = (np.arange(case["batch"]) + 0.5) / case["batch"]
    lo, hi = case["lo"], case["hi"]
    x = lo + u * (hi - lo) if case["dist"] == "uniform" else lo * (hi / lo) ** u
    x = np.clip(np.rint(x), lo, hi).astype(np.int64)
    return x if seed is None else np.random.RandomState(seed % (1 << 31)).permutation(x)


def _blocks(tokens):
    return -(-tokens // BLOCK)


def _seen(case, lens):
    """Per sequence: tokens that some new token sees, and pairs of new token and token seen."""
    n, W, S = case["n"], case["window"], case["sinks"]
    first = np.maximum(lens - n + 1 - W, 0)  # of the first new token's window
    tokens = lens - first + np.minimum(first, S)
    pairs = np.zeros(len(lens), np.int64)
    for i in range(n):
        end = np.maximum(lens - n + 1 + i, 0)
        start = np.maximum(end - W, 0)
        pairs += end - start + np.minimum(start, S)
    return tokens, pairs


def work(case):
    if case["op"] == "blocks":
        lens = _lens(case)
        new = np.minimum(lens, case["n"])
        rows, before, after = int(new.sum()), lens - new, lens - new + np.minimum(new, case["kept"])
        grown, back = int((_blocks(lens) - _blocks(before)).sum()), int((_blocks(lens) - _blocks(after)).sum())
        # ids read and written once each way; per call a length, a held count read and written; per row its
        # position, slot and block id
        return dict(bytes=float(8 * (grown + back) + 24 * len(lens) + 8 * rows + 4 * int((_blocks(lens) - before // BLOCK).sum())),
                    flops=float(rows))
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["op"] in ("rotary", "norm"):
        T, size = case["tokens"], 2 if case["dtype"] == "bf16" else 4
        rows = (T - T // 50) * (hq + hkv)
        passes, ops = (2, 0) if case["op"] == "rotary" else (3, 12 * d) if case["backward"] else (2, 4 * d)
        return dict(bytes=float(passes * rows * d * size + 4 * case["axes"] * T),
                    flops=float(rows * (3 * case["rotary_dim"] + ops)))
    lens = _lens(case)
    n, new = case["n"], int(np.minimum(lens, case["n"]).sum())
    if case["op"] == "store":
        return dict(bytes=float(new * (4 * hq * d + 8 * hkv * d) + 4 * (1 + case["axes"]) * new),
                    flops=float(new * (hq + hkv) * (3 * case["rotary_dim"] + 4 * d)))
    tokens, pairs = _seen(case, lens)
    return dict(bytes=float(tokens.sum() * hkv * 4 * d + 6 * new * hq * d + 4 * tokens.sum() / BLOCK + 4 * len(lens)),
                flops=float(4 * d * hq * pairs.sum()))


# ----------------------------------------------------------------- inputs --

def _table(lens, seed):
    """Block table (-1 past the ends) of contexts scattered over a pool a tenth larger than they need."""
    blocks = _blocks(lens)
    NB, width = int(math.ceil(1.1 * blocks.sum())), max(int(blocks.max()), 1)
    perm = np.random.RandomState((seed + 1) % (1 << 31)).permutation(NB).astype(np.int32)
    table, used = np.full((len(lens), width), -1, np.int32), 0
    for b, m in enumerate(blocks):
        table[b, :m] = perm[used:used + m]
        used += int(m)
    return table, NB, perm[used:]


def _positions(case, T, rng, seqs):
    """int32 [axes][T]: the running index on the first axis; on the others the same for text, and the row,
    column, ... of a patch for the middle third of every sequence."""
    axes, pos = case["axes"], []
    for start, count in seqs:
        p = np.tile(np.arange(start, start + count, dtype=np.int64), (axes, 1))
        a, b = count // 3, 2 * count // 3
        side = max(1, int(math.isqrt(max(1, b - a))))
        for x in range(1, axes):
            p[x, a:b] = start + a + (np.arange(b - a) // side ** (axes - 1 - x)) % side
        pos.append(p)
    return np.concatenate(pos, 1)[:, :T].astype(np.int32)


def _is_grad(case):
    return case["op"] == "norm" and case["backward"]


def _heads_common(case, state, gen):
    """Frequencies, the axis of every pair and the norms' weights."""
    dev, R = torch.device("cuda"), case["rotary_dim"]
    i = np.arange(R // 2)
    state["inv_freq"] = torch.from_numpy(case["base"] ** (-2.0 * i / R)).to(dev)
    # the axes' pairs: contiguous sections, or in turn where pairs are neighbours
    axis = i % case["axes"] if case["interleaved"] else i * case["axes"] // len(i)
    state["axis"] = torch.from_numpy(axis.astype(np.uint8)).to(dev)
    if case["op"] != "rotary":
        state["eps"] = 1e-6
        for name in ("q", "k"):
            w = 1 + 0.3 * torch.randn(case["head_dim"], generator=gen, device=dev)
            state[name + "_weight"] = w.to(torch.bfloat16 if case.get("dtype", "bf16") == "bf16" else torch.float32)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed + 7)
    rng = np.random.RandomState(seed % (1 << 31))
    state = dict(case)
    if case["op"] == "blocks":
        lens = _lens(case, seed)
        new = np.minimum(lens, case["n"])
        before, after = lens - new, lens - new + np.minimum(new, case["kept"])
        blocks = _blocks(lens)
        table, NB, spare = _table(lens, seed)
        # a running batch in steady state: what the rejected or released tokens' blocks were is on top of the stack
        held = _blocks(after)
        out = [table[b, held[b]:blocks[b]] for b in range(len(lens))]
        stack = np.concatenate([spare] + [np.concatenate(out)[::-1]]).astype(np.int32)
        free = np.full(NB, -1, np.int32)
        free[:len(stack)] = stack
        start = np.concatenate([[0], np.cumsum(new)])
        i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(dev)
        state.update(num_blocks=NB, table=i32(table), held=i32(held), free=i32(free), counts=i32([len(stack), 0]),
                     grown=i32(lens), after=i32(after), row_start=i32(start), rows=int(start[-1]),
                     longest=int(lens.max()))
        for name in ("positions", "slots"):
            state[name] = torch.full((state["rows"],), -7, dtype=torch.int32, device=dev)
        return state
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["op"] in ("rotary", "norm"):
        # a packed batch of sequences, padded to its size at the end
        T, seqs, total = case["tokens"], [], 0
        while total < T:
            seqs.append((rng.randint(1000), 1 + rng.randint(min(T, 4096))))
            total += seqs[-1][1]
        pos = _positions(case, T, rng, seqs)
        pos[:, T - T // 50:] = -1
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        # rows of the fused projection: a token's queries, keys and values side by side
        rows = torch.randn((T, hq + 2 * hkv, d), generator=gen, device=dev) * torch.exp2(torch.randn((T, 1, 1), generator=gen, device=dev))
        rows = rows.to(dtype)
        state.update(q=rows[:, :hq], k=rows[:, hq:hq + hkv], positions=torch.from_numpy(pos).to(dev))
        state["q_out"] = torch.zeros((T, hq, d), dtype=dtype, device=dev)
        state["k_out"] = torch.zeros((T, hkv, d), dtype=dtype, device=dev)
        if _is_grad(case):
            state["q_grad"] = torch.randn((T, hq, d), generator=gen, device=dev).to(dtype)
            state["k_grad"] = torch.randn((T, hkv, d), generator=gen, device=dev).to(dtype)
            for name in ("q", "k"):
                state[name + "_weight_grad"] = torch.zeros(d, dtype=torch.float32, device=dev)
        _heads_common(case, state, gen)
        return state
    lens = _lens(case, seed)
    B, n = case["batch"], case["n"]
    table, NB, _ = _table(lens, seed)
    if case["op"] == "store":
        new = np.minimum(lens, n)
        T = -(-int(new.sum()) // 8) * 8  # (a few rows of padding behind the last sequence)
        pos = np.full((case["axes"], T), -1, np.int32)
        pos[:, :int(new.sum())] = _positions(case, T, rng, [(x - m, m) for x, m in zip(lens, new)])
        slots = np.full(T, -1, np.int32)
        at, seq = pos[0, :int(new.sum())], np.repeat(np.arange(B), new)
        slots[:len(seq)] = table[seq, at // BLOCK] * BLOCK + at % BLOCK
        rows = torch.randn((T, hq + 2 * hkv, d), generator=gen, device=dev) * torch.exp2(torch.randn((T, 1, 1), generator=gen, device=dev))
        rows = rows.to(torch.bfloat16)
        state.update(q=rows[:, :hq], k=rows[:, hq:hq + hkv], v=rows[:, hq + hkv:],
                     positions=torch.from_numpy(pos).to(dev), slots=torch.from_numpy(slots).to(dev))
        state["q_out"] = torch.zeros((T, hq, d), dtype=torch.bfloat16, device=dev)
        state["k_cache"] = torch.zeros((NB, hkv, d // 8, BLOCK, 8), dtype=torch.bfloat16, device=dev)
        state["v_cache"] = torch.zeros((NB, hkv, BLOCK, d), dtype=torch.bfloat16, device=dev)
        _heads_common(case, state, gen)
        return state
    # Keys carry an offset per head and channel and a few strong channels, values differ in size from
    # token to token, as trained attention has.
    offset = torch.randn((hkv, 1, d), generator=gen, device=dev) * 0.5
    offset[:, :, ::37] *= 6
    k = (torch.randn((NB, hkv, BLOCK, d), generator=gen, device=dev) + offset).to(torch.bfloat16)
    v = torch.randn((NB, hkv, BLOCK, d), generator=gen, device=dev)
    v *= torch.exp2(torch.randn((NB, hkv, BLOCK, 1), generator=gen, device=dev))
    state.update(k_cache=k.view(NB, hkv, BLOCK, d // 8, 8).transpose(2, 3).contiguous(), v_cache=v.to(torch.bfloat16),
                 table=torch.from_numpy(table).to(dev), lens=torch.from_numpy(lens.astype(np.int32)).to(dev),
                 host_lens=lens, longest=int(lens.max()), softmax_scale=1.0 / math.sqrt(d))
    state["q"] = (torch.randn((B, n, hq, d), generator=gen, device=dev) * 1.5).to(torch.bfloat16)
    state["out"] = torch.zeros((B, n, hq, d), dtype=torch.float32, device=dev)
    return state


# -------------------------------------------------------------------- run --

def run(state):
    if own:
        return _own(state)
    plain = {"rotary": _heads, "norm": _grad if state.get("backward") else _heads, "store": _store, "window": _window, "blocks": _blocks_pass}
    return plain[state["op"]](state)


def _own(state):
    """The framework's calls, their arguments bound on a state's first pass as a serving loop binds them."""
    import paper_2405_11143_amd as pda

    op = state["op"]
    if "calls" not in state:
        heads = {}
        if op in ("rotary", "norm", "store"):
            heads["rotary"] = pda.make_rotary(state["inv_freq"], interleaved=state["interleaved"],
                                              backward=op == "rotary" and state["backward"])
            if state["axes"] > 1:
                heads["axes"] = pda.make_rotary_axes(state["axis"], state["axes"])
            if op != "rotary":
                heads["norm"] = pda.make_head_norm(state["q_weight"], state["k_weight"], eps=state["eps"])
            positions = state["positions"] if state["axes"] > 1 else state["positions"][0]
        if op == "rotary" or (op == "norm" and not state["backward"]):
            calls = [pda.bind_norm_rotary(state["q"], positions, k=state["k"], q_out=state["q_out"],
                                          k_out=state["k_out"], **heads)]
        elif op == "norm":
            calls = [pda.bind_norm_rotary_backward(state["q"], state["q_grad"], positions, k=state["k"],
                                                   k_grad=state["k_grad"], dq=state["q_out"], dk=state["k_out"],
                                                   dq_weight=state["q_weight_grad"], dk_weight=state["k_weight_grad"],
                                                   **heads)]
        elif op == "store":
            calls = [pda.bind_norm_rotary_append(state["q"], state["k"], state["v"], positions, state["slots"],
                                                 state["k_cache"], state["v_cache"], q_out=state["q_out"], **heads)]
        elif op == "window":
            calls = [pda.bind_decode_window(state["q"], state["k_cache"], state["v_cache"], state["table"],
                                            state["lens"], state["softmax_scale"], state["out"],
                                            window=state["window"], sinks=state["sinks"],
                                            max_context_len=state["longest"])]
        else:
            pool = pda.make_block_pool(state["table"], state["held"], state["free"], state["counts"])
            calls = [pda.bind_blocks_resize(pool, state["grown"], row_start=state["row_start"],
                                            positions=state["positions"], slots=state["slots"]),
                     pda.bind_blocks_resize(pool, state["after"])]
        state["calls"] = calls
    for call in state["calls"]:
        call()
    return _outputs(state)


def _outputs(state):
    op = state["op"]
    if op == "rotary" or (op == "norm" and not state["backward"]):
        return dict(q=state["q_out"], k=state["k_out"])
    if op == "norm":
        return dict(q=state["q_out"], k=state["k_out"], q_weight=state["q_weight_grad"], k_weight=state["k_weight_grad"])
    if op == "store":
        return dict(q=state["q_out"], k=state["k_cache"], v=state["v_cache"])
    if op == "window":
        return dict(out=state["out"])
    return dict(table=state["table"], held=state["held"], free=state["free"], counts=state["counts"],
                positions=state["positions"], slots=state["slots"])


def _turned(x, state, sign=1.0):
    """fp32 rows x [T, H, D] rotated at the state's positions [axes, T]."""
    R = state["rotary_dim"]
    angle = state["positions"].to(torch.float64)[state["axis"].long()].t() * state["inv_freq"]  # [T, R / 2]
    cos, sin = angle.cos().float()[:, None], (sign * angle.sin()).float()[:, None]
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if state["interleaved"] else (x[..., :R // 2], x[..., R // 2:R])
    c, e = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([c, e], -1).flatten(-2) if state["interleaved"] else torch.cat([c, e], -1)
    return torch.cat([turned, x[..., R:]], -1)


def _normed(x, weight, eps):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * weight.float()


def _heads(state):
    real = (state["positions"][0] >= 0)[:, None, None]
    for name in ("q", "k"):
        x = state[name].float()
        if state["op"] != "rotary":
            x = _normed(x, state[name + "_weight"], state["eps"])
        y = _turned(x, state, -1.0 if state["backward"] else 1.0).to(state[name].dtype)
        state[name + "_out"].copy_(torch.where(real, y, state[name + "_out"]))
    return _outputs(state)


def _grad(state):
    real = (state["positions"][0] >= 0)[:, None, None]
    for name in ("q", "k"):
        x = state[name].float()
        g = torch.where(real, _turned(state[name + "_grad"].float(), state, -1.0), 0.0)
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + state["eps"])
        unit = x * r
        gw = g * state[name + "_weight"].float()
        dx = r * (gw - unit * (gw * unit).mean(-1, keepdim=True))
        state[name + "_out"].copy_(torch.where(real, dx.to(state[name].dtype), state[name + "_out"]))
        state[name + "_weight_grad"].copy_((g * unit).sum((0, 1), dtype=torch.float64))
    return _outputs(state)


def _store(state):
    real = state["positions"][0] >= 0
    y = _turned(_normed(state["q"].float(), state["q_weight"], state["eps"]), state).to(torch.bfloat16)
    state["q_out"].copy_(torch.where(real[:, None, None], y, state["q_out"]))
    k = _turned(_normed(state["k"].float(), state["k_weight"], state["eps"]), state).to(torch.bfloat16)
    # (rows without a slot write what the first row writes, to its slot)
    row = torch.where(state["slots"] >= 0, torch.arange(len(state["slots"]), device=k.device), 0)
    slot = state["slots"][row].long()
    hkv, d = state["kv_heads"], state["head_dim"]
    state["k_cache"].permute(0, 3, 1, 2, 4)[slot // BLOCK, slot % BLOCK] = k[row].view(-1, hkv, d // 8, 8)
    state["v_cache"].transpose(1, 2)[slot // BLOCK, slot % BLOCK] = state["v"][row]
    return _outputs(state)


def _window(state):
    B, n, hq, d = state["q"].shape
    hkv, W, S = state["kv_heads"], state["window"], state["sinks"]
    G, lens, dev = hq // hkv, state["lens"].long(), state["q"].device
    # the tokens that some new token of the sequence sees: the first S and the first new token's window on
    T = min(state["longest"], S + W + n - 1)
    first = (lens - n + 1 - W).clamp(min=0)
    i = torch.arange(T, device=dev)
    sinks = first.clamp(max=S)[:, None]
    token = torch.where(i < sinks, i, i - sinks + first[:, None])  # [B, T]
    there = token < lens[:, None]
    token = torch.where(there, token, 0)
    ids = torch.gather(state["table"], 1, token // BLOCK).clamp(min=0).long()
    k = state["k_cache"].permute(0, 3, 1, 2, 4)[ids, token % BLOCK].float().view(B, T, hkv, d).permute(0, 2, 3, 1).contiguous()
    q = state["q"].float().view(B, n, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * G, d)
    s = torch.matmul(q, k) * state["softmax_scale"]
    del k
    at = (lens[:, None] - n + torch.arange(n, device=dev))[:, :, None]  # [B, n, 1]: the new tokens' positions
    t = token[:, None]
    seen = there[:, None] & (t <= at) & ((t > at - W) | (t < S))  # [B, n, T]
    s = s.view(B, hkv, n, G, T).masked_fill_(~seen[:, None, :, None], -math.inf).view(B, hkv, n * G, T)
    s = s.sub_(s.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = s.sum(-1, keepdim=True)
    v = state["v_cache"].transpose(1, 2)[ids, token % BLOCK].float().permute(0, 2, 1, 3).contiguous()
    out = torch.matmul(s, v) / total.clamp(min=1e-30)
    state["out"].copy_(out.view(B, hkv, n, G, d).permute(0, 2, 1, 3, 4).reshape(B, n, hq, d))
    return _outputs(state)


def _resize(state, lens):
    """Block tables for lengths `lens`, in elementary operations on the device."""
    table, held, free, counts = state["table"], state["held"].long(), state["free"], state["counts"]
    j = torch.arange(table.shape[1], device=table.device)
    need = (lens.long() + BLOCK - 1) // BLOCK
    # blocks put back: the first of them on top
    back = (j >= need[:, None]) & (j < held[:, None])
    count, back_rank = counts[0].long(), torch.cumsum(back.flatten(), 0).view_as(back) - 1
    back_total = back.sum()
    place = torch.where(back, count + back_total - 1 - back_rank, len(free)).flatten()
    stack = torch.cat([free, free.new_zeros(1)]).scatter(0, place, table.flatten())
    stack[-1] = 0
    count = count + back_total
    # blocks handed out, to the sequences whose running total is there
    want = (need - held).clamp(min=0)
    upto = torch.cumsum(want, 0)
    granted = upto <= count
    want = torch.where(granted, want, 0)
    before = torch.cumsum(want, 0) - want
    new = (j >= held[:, None]) & (j < (held + want)[:, None])
    source = count - 1 - (before[:, None] + j - held[:, None])
    table.copy_(torch.where(new, stack[source.clamp(0, len(free) - 1)], table))
    held.copy_(torch.where(need < held, need, held + want))
    state["held"].copy_(held)
    free.copy_(stack[:-1])
    counts[0] = count - want.sum()
    counts[1] = (upto[-1] - count).clamp(min=0)


def _map(state, lens):
    """Position and slot of every new token's row."""
    r = torch.arange(state["rows"], device=lens.device)
    start = state["row_start"].long()
    b = torch.searchsorted(start, r, right=True) - 1
    b = b.clamp(max=len(lens) - 1)
    at = lens.long()[b] - start[b + 1] + r
    real = (r < start[-1]) & (at >= 0)
    j = torch.where(real, at // BLOCK, 0)
    there = real & (j < state["held"][b])
    state["positions"].copy_(torch.where(real, at, -1))
    state["slots"].copy_(torch.where(there, state["table"][b, j].long() * BLOCK + at % BLOCK, -1))


def _blocks_pass(state):
    _resize(state, state["grown"])
    _map(state, state["grown"])
    _resize(state, state["after"])
    return _outputs(state)


# -------------------------------------------------------------- reference --

def _exact_turn(x, pos, state, sign):
    """Rows x [T, H, D] in 64 bits, each pair as a complex number turned by its own axis's angle."""
    R = state["rotary_dim"]
    angle = torch.stack([sign * pos[int(a)].double() * state["inv_freq"][i] for i, a in enumerate(state["axis"].cpu())], 1)
    turn = torch.polar(torch.ones_like(angle), angle)
    y = x.clone()
    first = slice(0, R, 2) if state["interleaved"] else slice(0, R // 2)
    second = slice(1, R, 2) if state["interleaved"] else slice(R // 2, R)
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn[:, None]
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_norm(x, weight, eps):
    return x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / x.shape[-1] + eps) * weight.double()


def _exact_blocks(state):
    """The pass on the host, one block id after the other."""
    table, held, free = (state[x].cpu().numpy().copy() for x in ("table", "held", "free"))
    count, short = int(state["counts"][0]), 0
    positions, slots = np.full(state["rows"], -1, np.int32), np.full(state["rows"], -1, np.int32)
    start = state["row_start"].cpu().numpy()
    for which in ("grown", "after"):
        lens = state[which].cpu().numpy()
        need, back, wanted, short = -(-lens // BLOCK), [], 0, 0
        for b in range(len(lens)):
            back += list(table[b, need[b]:held[b]])
            held[b] = min(held[b], need[b])
        free[count:count + len(back)] = back[::-1]
        count += len(back)
        there = count
        for b in range(len(lens)):
            more = int(need[b] - held[b])
            wanted += more
            if more > 0 and wanted <= there:
                table[b, held[b]:need[b]] = free[count - more:count][::-1]
                count, held[b] = count - more, need[b]
        short = max(0, wanted - there)
        for b in range(len(lens) if which == "grown" else 0):
            at, r = np.arange(lens[b] - (start[b + 1] - start[b]), lens[b]), slice(start[b], start[b + 1])
            positions[r] = at
            slots[r] = np.where(at // BLOCK < held[b], table[b, at // BLOCK] * BLOCK + at % BLOCK, -1)
    out = dict(table=table, held=held, free=free, counts=np.array([count, short], np.int32), positions=positions, slots=slots)
    return {name: torch.from_numpy(x).cuda() for name, x in out.items()}


def exact(case, seed):
    state = prepare(case, seed)
    f64, op = torch.float64, case["op"]
    if op == "blocks":
        return _exact_blocks(state)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    if op in ("rotary", "norm") and not _is_grad(case):
        out, real = {}, (state["positions"][0] >= 0)[:, None, None]
        for name in ("q", "k"):
            x = state[name].to(f64)
            if op == "norm":
                x = _exact_norm(x, state[name + "_weight"], state["eps"])
            out[name] = torch.where(real, _exact_turn(x, state["positions"], state, -1 if case["backward"] else 1), 0.0)
        return out
    if op == "norm":
        out, real = {}, state["positions"][0] >= 0
        for name in ("q", "k"):
            # y = W x / |x|' with |x|' = sqrt(mean x^2 + eps): dy/dx^T g, from the projection on x
            x, w = state[name].to(f64), state[name + "_weight"].to(f64)
            g = _exact_turn(state[name + "_grad"].to(f64), state["positions"], state, -1) * real[:, None, None]
            size = torch.sqrt((x ** 2).sum(-1, keepdim=True) / d + state["eps"])
            h = g * w
            along = (h * x).sum(-1, keepdim=True)
            out[name] = torch.where(real[:, None, None], h / size - x * along / (d * size ** 3), 0.0)
            out[name + "_weight"] = (g * x / size).flatten(0, 1).sum(0)
        return {x: out[x] for x in ("q", "k", "q_weight", "k_weight")}
    if op == "store":
        real = (state["positions"][0] >= 0)[:, None, None]
        rows = {}
        for name in ("q", "k"):
            x = _exact_norm(state[name].to(f64), state[name + "_weight"], state["eps"])
            rows[name] = _exact_turn(x, state["positions"], state, 1)
        out = dict(q=torch.where(real, rows["q"], 0.0), k=torch.zeros(state["k_cache"].shape, dtype=f64, device="cuda"),
                   v=torch.zeros(state["v_cache"].shape, dtype=f64, device="cuda"))
        r = torch.nonzero(state["slots"] >= 0)[:, 0]
        page, place = state["slots"][r].long() // BLOCK, state["slots"][r].long() % BLOCK
        for g in range(hkv):
            out["v"][page, g, place] = state["v"][r, g].to(f64)
            for c in range(d // 8):
                out["k"][page, g, c, place] = rows["k"][r, g, 8 * c:8 * c + 8]
        return out
    B, n, G, W, S = case["batch"], case["n"], hq // hkv, case["window"], case["sinks"]
    out = torch.zeros((B, n, hq, d), dtype=f64, device="cuda")
    for b, x in enumerate(int(x) for x in state["host_lens"]):
        i0 = max(0, n - x)  # new tokens before the context see nothing
        first = max(0, x - n + i0 + 1 - W)
        tokens = torch.cat([torch.arange(min(S, first), device="cuda"), torch.arange(first, x, device="cuda")])
        page, place = state["table"][b, tokens // BLOCK].long(), tokens % BLOCK
        kb = state["k_cache"][page, :, :, place].flatten(2).to(f64)  # [tokens, hkv, d]
        vb = state["v_cache"][page, :, place].to(f64)
        at = torch.arange(x - n + i0, x, device="cuda")[:, None]
        hidden = (tokens > at) | ((tokens <= at - W) & (tokens >= S))
        for g in range(hkv):
            qb = state["q"][b, i0:, g * G:(g + 1) * G].to(f64)
            w = (qb.reshape(-1, d) @ kb[:, g].T).view(n - i0, G, -1) * d ** -0.5
            w = torch.softmax(w.masked_fill(hidden[:, None], -math.inf), -1)
            out[b, i0:, g * G:(g + 1) * G] = (w.view(-1, len(tokens)) @ vb[:, g]).view(n - i0, G, d)
    return dict(out=out)
