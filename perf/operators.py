"""The operators of a model that generates with the attention-accumulated score, as a user's program calls them.

A case is a dict of plain values; "op" says which operator it takes:

  rotary   rotary positions of a projection's queries and keys (rotary), or the gradients taken back through them.
  kv       new keys, values and modality scores into a paged cache and back out of it (kv_write, kv_read), as a
           chunked prefill does before it attends to what the cache holds.
  decode   attention of one new token per sequence over a paged cache, with the modality scores as two more value
           channels (attention_scores_decode).

Sizes are those of the attention of this repository's tests and benchmark (16 heads of 128; 32 heads over 8 or 4 KV
heads of 64 or 128), batches of 1 to 256 sequences, caches of one token to 131072, pages of 16 to 256 tokens.
With `own` false the operators are computed in their plain form from elementary torch operations in float32 (angles
in float64); with `own` true by the framework. Inputs are drawn on the GPU from the seed alone; sequence lengths
follow from the case.
"""
import math

import torch

own = False

DEV = "cuda:0"
GOLDEN = 0.6180339887498949
BYTES_MOST = 4.0e9  # of a drawn decode's cache; the largest listed one reads 4.3e9


def listed():
    return [
        # one step of a few chats: the smallest call, where latency is all
        dict(name="rotary-step-8", op="rotary", tokens=8, heads=16, kv_heads=16, head_dim=128, rot_dim=128,
             layout="half", scaling="none", factor=1.0, dtype="bf16", backward=False, start=2000),
        # prefill of a long-context model: interleaved pairs, frequencies scaled by parts, positions far out
        dict(name="rotary-long-16384", op="rotary", tokens=16384, heads=32, kv_heads=8, head_dim=128, rot_dim=128,
             layout="interleaved", scaling="by_parts", factor=32.0, dtype="bf16", backward=False, start=100000),
        # a float32 run (parity check, small training) of a model that rotates half of each head, odd batch
        dict(name="rotary-part-f32-4099", op="rotary", tokens=4099, heads=32, kv_heads=4, head_dim=64, rot_dim=32,
             layout="half", scaling="linear", factor=4.0, dtype="f32", backward=False, start=0),
        # the gradient of a training batch's queries and keys
        dict(name="rotary-grad-8113", op="rotary", tokens=8113, heads=16, kv_heads=16, head_dim=128, rot_dim=128,
             layout="half", scaling="ntk", factor=8.0, dtype="bf16", backward=True, start=0),
        # one step of a batch into a bf16 cache
        dict(name="kv-step-bf16-32", op="kv", seqs=32, tokens=32, step=True, kv_heads=16, head_dim=128, kind="bf16",
             dtype="bf16", page=16, past=1000, pad=0),
        # one step of a large batch into an 8-bit cache, some slots of the batch unused
        dict(name="kv-step-e4m3-256", op="kv", seqs=256, tokens=256, step=True, kv_heads=8, head_dim=128, kind="e4m3",
             dtype="bf16", page=32, past=3000, pad=0),
        # a chunk of sixteen prompts into an 8-bit cache behind what is there already, rows of padding behind the last
        dict(name="kv-prefill-e4m3-16384", op="kv", seqs=16, tokens=16384, step=False, kv_heads=8, head_dim=128,
             kind="e4m3", dtype="bf16", page=64, past=2000, pad=37),
        # float32 activations into a bf16 cache, ragged prompts, heads of 64
        dict(name="kv-prefill-f32-7001", op="kv", seqs=5, tokens=7001, step=False, kv_heads=4, head_dim=64,
             kind="bf16", dtype="f32", page=16, past=0, pad=0),
        # the first words of one short chat
        dict(name="decode-1x37", op="decode", seqs=1, short=37, long=37, empty=0, heads=16, kv_heads=16, head_dim=128,
             kind="bf16", page=16),
        # one chat over a whole book: the length has to be split over the chip
        dict(name="decode-1x131072", op="decode", seqs=1, short=131072, long=131072, empty=0, heads=32, kv_heads=8,
             head_dim=128, kind="bf16", page=64),
        # a serving batch of unequal lengths on an 8-bit cache, three of its slots unused
        dict(name="decode-64-e4m3", op="decode", seqs=64, short=200, long=20000, empty=3, heads=32, kv_heads=8,
             head_dim=128, kind="e4m3", page=32),
        # the largest: a KV head per query head, a full batch of image prompts
        dict(name="decode-128-bf16", op="decode", seqs=128, short=2500, long=6500, empty=0, heads=16, kv_heads=16,
             head_dim=128, kind="bf16", page=16),
    ]


# ---------------------------------------------------------------- drawn cases

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "kv", "decode"])
    head_dim = rng.choice([64, 128])
    heads, kv_heads = rng.choice([(16, 16), (32, 8), (32, 4), (8, 1), (12, 4), (40, 2)])
    if op == "rotary":
        return dict(op=op, tokens=_log_int(rng, 1, 12000), heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                    rot_dim=rng.choice([head_dim, head_dim // 2, head_dim // 4, head_dim // 2 + 2]),
                    layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "ntk", "by_parts"]), factor=round(rng.uniform(1.5, 40.0), 2),
                    dtype=rng.choice(["bf16", "bf16", "f32"]), backward=rng.random() < 0.4,
                    start=rng.choice([0, _log_int(rng, 1, 1000000)]))
    if op == "kv":
        step = rng.random() < 0.4
        seqs = _log_int(rng, 1, 256) if step else _log_int(rng, 1, 32)
        tokens = seqs if step else max(seqs, _log_int(rng, 10, 16000))
        return dict(op=op, seqs=seqs, tokens=tokens, step=step, kv_heads=kv_heads, head_dim=head_dim,
                    kind=rng.choice(["bf16", "e4m3"]), dtype=rng.choice(["bf16", "bf16", "f32"]),
                    page=rng.choice([16, 32, 64, 128, 256]), past=rng.choice([0, _log_int(rng, 1, 4000)]),
                    pad=0 if step else rng.choice([0, rng.randrange(1, 100)]))
    kind = rng.choice(["bf16", "e4m3"])
    row = kv_heads * head_dim * 2 * (2 if kind == "bf16" else 1)
    seqs = _log_int(rng, 1, 256)
    most = max(1, min(131072, int(BYTES_MOST / row / seqs)))
    long = _log_int(rng, 1, most)
    short = _log_int(rng, 1, long)
    return dict(op=op, seqs=seqs, short=short, long=long, empty=rng.choice([0, min(seqs - 1, rng.randrange(0, 4))]),
                heads=heads, kv_heads=kv_heads, head_dim=head_dim, kind=kind, page=rng.choice([16, 32, 64, 128, 256]))


# ---------------------------------------------------------------- sizes that follow from the case

def _lengths(case):
    """Keys of every sequence of a decode case: spread over [short, long] by their logarithm, the first ones empty."""
    lo, hi = case["short"], case["long"]
    out = [max(1, int(round(lo * (hi / lo) ** ((GOLDEN * (b + 1)) % 1.0)))) for b in range(case["seqs"])]
    return [0 if b < case["empty"] else n for b, n in enumerate(out)]


def _chunks(case):
    """New tokens of every sequence of a kv case, and its length with them. In a step the last of more than 100
    sequences are slots of the batch that no chat uses: length 0, nothing written or read."""
    n = case["seqs"]
    if case["step"]:
        new = [1] * n
    else:
        share = [0.25 + (GOLDEN * (b + 1)) % 1.0 for b in range(n)]
        new = [1 + int((case["tokens"] - n) * s / sum(share)) for s in share]
        new[-1] += case["tokens"] - sum(new)
    past = [int(case["past"] * (0.5 + (GOLDEN * (b + 3)) % 1.0)) for b in range(n)]
    total = [a + b for a, b in zip(new, past)]
    if case["step"] and n > 100:
        total[-3:] = [0, 0, 0]
    return new, total


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def work(case):
    if case["op"] == "rotary":
        size = 2 if case["dtype"] == "bf16" else 4
        elems = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["head_dim"]
        rotated = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["rot_dim"]
        return {"bytes": 2 * elems * size + 4 * case["tokens"], "flops": 3 * rotated}
    if case["op"] == "kv":
        # keys, values and scores read once, their cached form written, read again, and written out as bf16
        rows = 2 * case["tokens"] * case["kv_heads"]
        held = case["head_dim"] * 2 if case["kind"] == "bf16" else case["head_dim"] + 1
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": rows * (case["head_dim"] * (size + 2) + 2 * held) + 4 * 8 * case["tokens"],
                "flops": 2 * rows * case["head_dim"]}
    keys = sum(_lengths(case))
    held = case["head_dim"] * 2 if case["kind"] == "bf16" else case["head_dim"] + 1
    rows = case["seqs"] * case["heads"]
    return {"bytes": keys * (2 * case["kv_heads"] * held + 8) + rows * (case["head_dim"] * 4 + 8),
            "flops": keys * case["heads"] * (4 * case["head_dim"] + 4)}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV, dtype=dtype)


def _pages(case, total, g):
    """Block table [sequences, most pages] (-1 behind a sequence's last page) in a random order of pages, and their number."""
    page = case["page"]
    need = [-(-n // page) for n in total]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(total), max(1, max(need))), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, n_pages


def _inputs(case, seed):
    """A case's inputs as plain tensors."""
    g = _gen(seed)
    if case["op"] == "rotary":
        T, H, Hkv, dh, dt = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"], _dtype(case["dtype"])
        if case["backward"]:
            q, k = _randn(g, T, H, dh, dtype=dt), _randn(g, T, Hkv, dh, dtype=dt)
        else:  # views into one projection's output, as a fused projection leaves them
            qkv = _randn(g, T, H + 2 * Hkv, dh, dtype=dt)
            q, k = qkv[:, :H], qkv[:, H:H + Hkv]
        if T <= 256:  # a step: every sequence at its own position
            pos = torch.randint(case["start"], 2 * case["start"] + 100, (T,), generator=g, device=DEV)
        else:
            pos = case["start"] + torch.arange(T, device=DEV) % 5000
        return dict(q=q, k=k, positions=pos.to(torch.int32))
    if case["op"] == "kv":
        new, total = _chunks(case)
        rows, Hkv, dh, dt = case["tokens"] + case["pad"], case["kv_heads"], case["head_dim"], _dtype(case["dtype"])
        kv = _randn(g, rows, 2 * Hkv, dh, dtype=dt)
        kv *= torch.exp(_randn(g, rows, 2 * Hkv, 1)).to(dt)  # rows of unequal size
        table, n_pages = _pages(case, total, g)
        score = torch.rand(rows, 1, generator=g, device=DEV)
        offsets = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32, device=DEV)
        return dict(k=kv[:, :Hkv], v=kv[:, Hkv:], m=torch.cat([score, 1 - score], 1).contiguous(), table=table,
                    n_pages=n_pages, lengths=torch.tensor(total, dtype=torch.int32, device=DEV),
                    offsets=None if case["step"] else offsets)
    lengths = _lengths(case)
    H, Hkv, dh, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    table, n_pages = _pages(case, lengths, g)
    shape = (n_pages, Hkv, page, dh)
    out = dict(table=table, lengths=torch.tensor(lengths, dtype=torch.int32, device=DEV), n_pages=n_pages)
    for name in ("k", "v"):
        if case["kind"] == "bf16":
            out[name] = _randn(g, *shape, dtype=torch.bfloat16)
        else:
            codes = torch.empty(shape, dtype=torch.uint8, device=DEV)
            for a in range(0, n_pages, 4096):
                x = _randn(g, *codes[a:a + 4096].shape) * 64.0
                codes[a:a + 4096] = x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
            out[name] = codes
            out[name + "_scale"] = torch.randint(120, 123, shape[:3], generator=g, device=DEV).to(torch.uint8)
    score = torch.rand(n_pages, page, generator=g, device=DEV)
    out["m"] = torch.stack([score, 1 - score], 1).contiguous()
    qkv = _randn(g, case["seqs"], H + 2 * Hkv, dh, dtype=torch.bfloat16)
    out["q"] = 2.0 * qkv[:, :H] if case["seqs"] % 2 else (2.0 * qkv)[:, :H]  # dense, or a view into the projection
    return out


def _rope(case):
    """Arguments of a case's rotary positions."""
    return dict(head_dim=case["head_dim"], rot_dim=case["rot_dim"], layout=case["layout"], scaling=case["scaling"],
                base=10000.0, factor=case["factor"], original_len=4096, beta_fast=32.0, beta_slow=1.0)


def prepare(case, seed):
    state = dict(case=case, **_inputs(case, seed))
    if own:
        from paper_2604_23996_amd import smoes as S
    if case["op"] == "rotary":
        state["q_out"] = torch.empty(state["q"].shape, dtype=state["q"].dtype, device=DEV)
        state["k_out"] = torch.empty(state["k"].shape, dtype=state["k"].dtype, device=DEV)
        if own:
            state["plan"] = S.RotaryPlan(S.RotarySpec(**_rope(case)), device=DEV)
        else:
            state["freqs"], state["amplitude"] = _plain_frequencies(**_rope(case))
        return state
    if case["op"] == "kv":
        rows, Hkv, dh, page = case["tokens"] + case["pad"], case["kv_heads"], case["head_dim"], case["page"]
        for name in ("k_out", "v_out"):
            state[name] = torch.zeros(rows, Hkv, dh, dtype=torch.bfloat16, device=DEV)
        state["m_out"] = torch.zeros(rows, 2, device=DEV)
        if own:
            state["cache"] = S.KVCache(state["n_pages"], page, Hkv, dh, kind=case["kind"], device=DEV)
        else:
            for name in ("k", "v"):
                dt = torch.bfloat16 if case["kind"] == "bf16" else torch.uint8
                state[name + "_pages"] = torch.zeros(state["n_pages"], Hkv, page, dh, dtype=dt, device=DEV)
                state[name + "_scale"] = torch.zeros(state["n_pages"], Hkv, page, dtype=torch.uint8, device=DEV)
            state["m_pages"] = torch.zeros(state["n_pages"], 2, page, device=DEV)
        return state
    if own:
        state["cache"] = S.KVCache(state["n_pages"], case["page"], case["kv_heads"], case["head_dim"],
                                   kind=case["kind"], device=DEV, k=state["k"], v=state["v"],
                                   k_scale=state.get("k_scale"), v_scale=state.get("v_scale"), m=state["m"])
        n = S.attention_decode_workspace_bytes(state["cache"], case["seqs"], case["heads"])
        state["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV)
        state["o"] = torch.empty(case["seqs"], case["heads"], case["head_dim"], dtype=torch.bfloat16, device=DEV)
        state["m_heads"] = torch.empty(case["seqs"], case["heads"], 2, device=DEV)
    else:
        state["lens"] = _lengths(case)
    return state


# ---------------------------------------------------------------- the passes

def run(state):
    case = state["case"]
    if own:
        from paper_2604_23996_amd import smoes as S
        if case["op"] == "rotary":
            return S.rotary(state["plan"], state["q"], state["k"], positions=state["positions"],
                            backward=case["backward"], q_out=state["q_out"], k_out=state["k_out"])
        if case["op"] == "kv":
            S.kv_write(state["cache"], state["table"], state["lengths"], state["k"], state["v"], state["m"],
                       sample_offsets=state["offsets"])
            return S.kv_read(state["cache"], state["table"], state["lengths"], sample_offsets=state["offsets"],
                             k=state["k_out"], v=state["v_out"], m=state["m_out"])
        return S.attention_scores_decode(state["cache"], state["table"], state["lengths"], state["q"], o=state["o"],
                                         m_heads=state["m_heads"], workspace=state["workspace"])
    if case["op"] == "rotary":
        return _plain_rotary(state)
    if case["op"] == "kv":
        return _plain_kv(state)
    return _plain_decode(state)


# ---------------------------------------------------------------- plain forms

def _plain_frequencies(head_dim, rot_dim, layout, scaling, base, factor, original_len, beta_fast, beta_slow):
    """Radians per position of each rotated pair, and the amplitude."""
    i = torch.arange(0, rot_dim, 2, dtype=torch.float64, device=DEV)
    if scaling == "ntk":
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = base ** (-i / rot_dim)
    if scaling == "linear":
        f = f / factor
    if scaling != "by_parts":
        return f, 1.0
    turns = original_len * f / (2 * math.pi)
    keep = ((turns - beta_slow) / (beta_fast - beta_slow)).clamp(0, 1)
    return keep * f + (1 - keep) * f / factor, 1 + 0.1 * math.log(factor)


def _plain_rotary(state):
    case = state["case"]
    r, a = case["rot_dim"], state["amplitude"]
    angle = state["positions"].double()[:, None] * state["freqs"]
    if case["backward"]:
        angle = -angle
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    for x, y in ((state["q"], state["q_out"]), (state["k"], state["k_out"])):
        if case["layout"] == "half":
            i, j = slice(0, r // 2), slice(r // 2, r)
        else:
            i, j = slice(0, r, 2), slice(1, r, 2)
        x0, x1 = x[..., i].float(), x[..., j].float()
        y[..., i] = (a * (x0 * cos - x1 * sin)).to(y.dtype)
        y[..., j] = (a * (x0 * sin + x1 * cos)).to(y.dtype)
        y[..., r:] = x[..., r:]
    return state["q_out"], state["k_out"]


def _plain_kv(state):
    case, page = state["case"], state["case"]["page"]
    n, rows = case["seqs"], case["tokens"]
    seq = torch.arange(n, device=DEV)
    lengths = state["lengths"].long()
    if state["offsets"] is None:
        pos = lengths - 1
    else:
        offsets = state["offsets"].long()
        new = offsets[1:] - offsets[:-1]
        seq = torch.repeat_interleave(seq, new, output_size=rows)
        pos = lengths[seq] - new[seq] + torch.arange(rows, device=DEV) - offsets[seq]
    keep = slice(0, n - 3) if case["step"] and n > 100 else slice(0, rows)  # the slots of the batch in use
    seq, pos = seq[keep], pos[keep]
    pid, slot = state["table"][seq, pos // page].long(), pos % page
    for name in ("k", "v"):
        x = state[name][:rows][keep].float()
        pages = state[name + "_pages"]
        if case["kind"] == "bf16":
            pages[pid, :, slot] = x.to(torch.bfloat16)
            back = pages[pid, :, slot]
        else:
            # the smallest power of two (2^-117 at least) that brings the row's largest value to 448 = 0.875 * 2^9 or less
            mant, ex = torch.frexp(x.abs().amax(-1))
            e = torch.where(mant > 0.875, ex - 8, ex - 9).clamp(min=-117)
            e = torch.where(mant == 0, torch.zeros_like(e), e)
            codes = torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn)
            pages[pid, :, slot] = codes.view(torch.uint8)
            state[name + "_scale"][pid, :, slot] = (e + 127).to(torch.uint8)
            e = state[name + "_scale"][pid, :, slot].int() - 127
            back = torch.ldexp(pages[pid, :, slot].view(torch.float8_e4m3fn).float(), e[..., None])
        state[name + "_out"][:rows][keep] = back.to(torch.bfloat16)
    state["m_pages"][pid, :, slot] = state["m"][:rows][keep]
    state["m_out"][:rows][keep] = state["m_pages"][pid, :, slot]
    return state["k_out"], state["v_out"], state["m_out"]


def _plain_decode(state):
    case, page = state["case"], state["case"]["page"]
    H, Hkv, dh = case["heads"], case["kv_heads"], case["head_dim"]
    o = torch.zeros(case["seqs"], H, dh, dtype=torch.bfloat16, device=DEV)
    m_heads = torch.zeros(case["seqs"], H, 2, device=DEV)
    for b, n in enumerate(state["lens"]):
        if n == 0:
            continue
        at = state["table"][b, :-(-n // page)].long()
        kv = []
        for name in ("k", "v"):
            x = state[name][at]
            if case["kind"] == "e4m3":
                e = state[name + "_scale"][at].int() - 127
                x = torch.ldexp(x.view(torch.float8_e4m3fn).float(), e[..., None])
            kv.append(x.float().transpose(0, 1).reshape(Hkv, -1, dh)[:, :n])
        m = state["m"][at].transpose(1, 2).reshape(-1, 2)[:n]
        s = torch.matmul(state["q"][b].float().view(Hkv, H // Hkv, dh), kv[0].transpose(1, 2)) / math.sqrt(dh)
        p = torch.exp(s - s.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        o[b] = torch.matmul(p, kv[1]).view(H, dh).to(torch.bfloat16)
        m_heads[b] = torch.matmul(p, m).view(H, 2)
    return o, m_heads


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    x = _inputs(case, seed)
    if case["op"] == "rotary":
        return _exact_rotary(case, x)
    if case["op"] == "kv":
        return _exact_kv(case, x)
    return _exact_decode(case, x)


def _exact_rotary(case, x):
    """Each pair as a complex number, times amplitude * e^(i position frequency) (its conjugate for the gradient)."""
    r, s, f, amplitude = case["rot_dim"], case["factor"], [], 1.0
    for i in range(r // 2):
        rate = math.exp(-2 * i / r * math.log(10000.0))
        if case["scaling"] == "linear":
            rate /= s
        elif case["scaling"] == "ntk":
            rate = math.exp(-2 * i / r * (math.log(10000.0) + r / (r - 2) * math.log(s)))
        elif case["scaling"] == "by_parts":
            keep = min(1.0, max(0.0, (4096 * rate / (2 * math.pi) - 1.0) / 31.0))
            rate = rate / s + keep * (rate - rate / s)
            amplitude = 1 + 0.1 * math.log(s)
        f.append(-rate if case["backward"] else rate)
    angle = x["positions"].double()[:, None] * torch.tensor(f, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.full_like(angle, amplitude), angle)[:, None]
    out = []
    for t in (x["q"].double(), x["k"].double()):
        rot, rest = t[..., :r], t[..., r:]
        if case["layout"] == "half":
            z = torch.complex(rot[..., :r // 2].contiguous(), rot[..., r // 2:].contiguous()) * turn
            out.append(torch.cat([z.real, z.imag, rest], -1))
        else:
            z = torch.view_as_complex(rot.reshape(*rot.shape[:-1], r // 2, 2).contiguous()) * turn
            out.append(torch.cat([torch.view_as_real(z).flatten(-2), rest], -1))
    return tuple(out)


def _exact_kv(case, x):
    """What a row stands for after the cache: itself, or on the grid of e4m3 (three bits behind the leading one, exponents
    from -6) times the row's power of two."""
    new, total = _chunks(case)
    held = torch.zeros(case["tokens"] + case["pad"], dtype=torch.bool, device=DEV)
    at = 0
    for n, length in zip(new, total):
        held[at:at + n] = length >= n
        at += n
    out = []
    for t in (x["k"].double(), x["v"].double()):
        if case["kind"] == "e4m3":
            top = t.abs().amax(-1, keepdim=True)
            e = torch.ceil(torch.log2(top / 448.0))
            e = torch.where(top > 448.0 * torch.exp2(e), e + 1, e)
            e = torch.where(top <= 224.0 * torch.exp2(e), e - 1, e)
            s = torch.where(top > 0, torch.exp2(e.clamp(min=-117.0)), torch.ones_like(top))
            y = t / s
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
            t = torch.round(y / step) * step * s  # ties to even
        out.append(torch.where(held[:, None, None], t, torch.zeros_like(t)))
    out.append(torch.where(held[:, None], x["m"].double(), torch.zeros_like(x["m"].double())))
    return tuple(out)


def _exact_decode(case, x):
    H, Hkv, dh, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    o = torch.zeros(case["seqs"], H, dh, dtype=torch.float64, device=DEV)
    m_heads = torch.zeros(case["seqs"], H, 2, dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lengths(case)):
        if n == 0:
            continue
        j = torch.arange(n, device=DEV)
        pid, slot = x["table"][b].long()[j // page], j % page
        rows = []
        for name in ("k", "v"):
            t = x[name][pid, :, slot]  # [keys, KV heads, head_dim]
            if case["kind"] == "e4m3":
                t = t.view(torch.float8_e4m3fn).double() * torch.exp2(x[name + "_scale"][pid, :, slot].double() - 127)[..., None]
            rows.append(t.double())
        score = x["m"][pid, :, slot].double()
        for h in range(Hkv):
            mine = slice(h * (H // Hkv), (h + 1) * (H // Hkv))
            s = torch.mm(x["q"][b, mine].double(), rows[0][:, h].t().contiguous()) / math.sqrt(dh)
            p = torch.softmax(s, -1)
            o[b, mine] = torch.mm(p, rows[1][:, h].contiguous())
            m_heads[b, mine] = torch.mm(p, score)
    return o, m_heads
