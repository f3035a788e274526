"""The operators around keys and values in 8 bits, as measurable cases.

Four calls, in the order a serving program makes them: a projection's rows are normed per head, rotated and laid out
(`rotate`); the fixed context is held in 8 bits with a scale per 64 keys and head (`quantize`); new tokens are appended to a
paged 8-bit cache (`append`); a decode step attends to kept ranges of the fixed context and to the paged cache (`attend`).
Data are drawn on the GPU from the seed alone.
"""
import math
import random

import torch

own = False

D = 128
BLOCK = 64                                   # keys of the fixed context that share a scale
SM_SCALE = float(torch.tensor(1.0 / math.sqrt(D), dtype=torch.float32))
EPS = float(torch.tensor(1e-6, dtype=torch.float32))
E_MIN, E_MAX = -64, 64                       # exponents of a block's scale
F8, F16, F32, F64, I32, U8 = torch.float8_e4m3fn, torch.float16, torch.float32, torch.float64, torch.int32, torch.uint8


def _rotate(name, B, Lq, H, G, norm, rot, pairs, n_pos):
    return dict(name=name, kind="rotate", B=B, Lq=Lq, H=H, G=G, norm=norm, rot=rot, pairs=pairs, n_pos=n_pos)


def _append(name, B, T, H, G, norm, rot, pairs, n_pos, page, old, pad=0):
    """T tokens in all, dealt at random over the B sequences (T == B: one each); `old`: the most tokens a sequence has so far."""
    return dict(name=name, kind="append", B=B, T=T, H=H, G=G, norm=norm, rot=rot, pairs=pairs, n_pos=n_pos, page=page, old=old, pad=pad)


def _quantize(name, B, H, L, perm):
    return dict(name=name, kind="quantize", B=B, H=H, L=L, perm=perm)


def _attend(name, B, H, G, L, C, keep, user, page, one_set=False):
    """keep: share of the fixed context's keys that a row keeps on average (C = 0: no fixed context); user: the longest sequence."""
    return dict(name=name, kind="attend", B=B, H=H, G=G, L=L, C=C, keep=keep, user=user, page=page, one_set=one_set)


def listed():
    return [
        # The rows of one generated token of a model with normed heads, 32 query heads over 8 K/V heads: launch latency.
        _rotate("rotate_token", 1, 1, 8, 4, True, 128, "halves", 65536),
        # A 1024-token prompt of a 7B-shaped layer (no norms): what the prefill steps take as q, K_user and V_user.
        _rotate("rotate_prompt", 1, 1024, 32, 1, False, 128, "halves", 65536),
        # A 32K fixed context on its way to the clustering, grouped heads with norms.
        _rotate("rotate_context", 1, 32768, 8, 4, True, 128, "halves", 65536),
        # One token of one sequence into its page: the smallest append.
        _append("append_token", 1, 1, 32, 1, False, 128, "halves", 65536, 64, 512),
        # A decode step of 64 sequences, grouped heads with norms, pages of 16 tokens.
        _append("append_batch", 64, 64, 8, 4, True, 128, "halves", 65536, 16, 2048),
        # Prompts of uneven length that arrive together, behind what their sequences hold, with a padded end.
        _append("append_prompts", 13, 16384, 8, 4, True, 64, "adjacent", 65536, 64, 700, 5),
        # A short context of few heads, sorted already.
        _quantize("quantize_4k", 1, 4, 4096, False),
        # The 32K context of 32 heads through the order that the clustering found.
        _quantize("quantize_32k", 1, 32, 32768, True),
        # One token over a short context with few heads: launches and dependent reads.
        _attend("attend_4k", 1, 4, 1, 4096, 64, 1 / 4, 128, 64),
        # One token of a 7B-shaped layer over a 32K context.
        _attend("attend_32k", 1, 32, 1, 32768, 1024, 1 / 8, 512, 64),
        # A full batch over one shared prefix, every sequence with a selection of its own.
        _attend("attend_shared_b16", 16, 32, 1, 32768, 1024, 1 / 8, 256, 16),
        # Eight sequences of grouped heads, one kept set per K/V head, long and uneven answers behind a 128K context.
        _attend("attend_grouped_b8", 8, 8, 4, 131072, 4096, 1 / 16, 16384, 64, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "append", "append", "quantize", "attend", "attend", "attend"])
    H, G = rng.choice([(1, 8), (2, 16), (4, 1), (5, 3), (8, 4), (8, 5), (12, 1), (20, 1), (32, 1)])
    rope = dict(norm=rng.random() < 0.5, rot=rng.choice([128, 128, 96, 64, 32]), pairs=rng.choice(["halves", "adjacent"]),
                n_pos=_log_int(rng, 4096, 131072))
    if kind == "rotate":
        B, heads = rng.choice([1, 1, 2, 5]), H * G + 2 * H
        return dict(kind=kind, B=B, Lq=_log_int(rng, 1, 32768 * 48 // (B * heads)), H=H, G=G, **rope)
    if kind == "append":
        B = _log_int(rng, 1, 100)
        T = B if rng.random() < 0.5 else max(B, _log_int(rng, 16, 16384 * 48 // (H * G + 2 * H)))
        return dict(kind=kind, B=B, T=T, H=H, G=G, **rope, page=rng.choice([16, 32, 64]), old=_log_int(rng, 1, 2000), pad=rng.choice([0, 0, 7]))
    if kind == "quantize":
        B = rng.choice([1, 1, 3])
        return dict(kind=kind, B=B, H=H, L=_log_int(rng, 500, 32768 * 32 // (B * H)), perm=rng.random() < 0.6)
    B, one_set = _log_int(rng, 1, 16), G > 1 and rng.random() < 0.5
    rows = B * H * (1 if one_set else G)
    L = _log_int(rng, 500, 131072)
    user = _log_int(rng, 1, min(16384, 1_500_000 // rows))
    keep = min(round(rng.uniform(0.03, 0.3), 3), 1_000_000 / rows / L)
    C = 0 if rng.random() < 0.2 else max(8, min(16384, L // rng.randint(20, 64)))
    return dict(kind=kind, B=B, H=H, G=G, L=L, C=C, keep=keep, user=user, page=rng.choice([16, 32, 64]), one_set=one_set)


# ---------------------------------------------------------------------------------------------------------------------
# Inputs.
# ---------------------------------------------------------------------------------------------------------------------
def _table(n_pos, rot):
    """cos and sin of every position and pair, base 10000: f32 [n_pos, rot / 2, 2]."""
    freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=F64, device="cuda") / rot)
    a = torch.arange(n_pos, dtype=F64, device="cuda").unsqueeze(1) * freq
    return torch.stack([a.cos(), a.sin()], 2).float().contiguous()


def _projection(case, g, T):
    """The rows of one fused projection [T, (q heads, k heads, v heads), 128] and the norms' weights."""
    H, G = case["H"], case["G"]
    x = torch.randn(T, H * G + 2 * H, D, generator=g, device="cuda").half()
    w = [(1 + 0.1 * torch.randn(D, generator=g, device="cuda")).half() if case["norm"] else None for _ in range(2)]
    return dict(q=x[:, :H * G], k=x[:, H * G:H * G + H], v=x[:, H * G + H:], w_q=w[0], w_k=w[1],
                table=_table(case["n_pos"], case["rot"]), adjacent=case["pairs"] == "adjacent")


def _pages(case, g, lengths, spare, old=False):
    """A pool with a page table for sequences of these lengths, `spare` pages unused; codes of whole pages, filled or not."""
    P, H, B = case["page"], case["H"], case["B"]
    width = max(1, max(-(-n // P) for n in lengths))
    used = B * width
    ids = torch.randperm(used + spare, generator=g, device="cuda")[:used].view(B, width).int().contiguous()
    codes = [(64 * torch.randn(used + spare, H, P, D, generator=g, device="cuda")).clamp(-448, 448).to(F8) for _ in range(2)]
    # scales about those of values ~ N(0, 1), so that what is appended raises some of them
    scales = [torch.exp2(torch.randint(-9 if old else -7, -5, (used + spare, H), generator=g, device="cuda").float()) for _ in range(2)]
    return dict(cK=codes[0], cV=codes[1], cks=scales[0], cvs=scales[1], pages=ids)


def _dealt(case):
    """How many tokens every sequence has so far and gets (plain integers, the case's own)."""
    B, T = case["B"], case["T"]
    r = random.Random(B * 1000003 + T)
    old = [r.randint(0, case["old"]) for _ in range(B)]
    if T == B:
        return old, [1] * B
    cuts = sorted(r.randint(0, T) for _ in range(B - 1))
    return old, [hi - lo for lo, hi in zip([0] + cuts, cuts + [T])]


def _shares(case):
    """The share of the keys that each row keeps: uneven, and `keep` on average; rows of (sequence, head[, query head])."""
    n = case["B"] * case["H"] * (1 if case["one_set"] else case["G"])
    f = [0.2 + 1.6 * ((r + 1) * 0.6180339887498949 % 1.0) for r in range(n)]
    scale = case["keep"] * n / sum(f)
    return [min(1.0, v * scale) for v in f]


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind = case["kind"]
    if kind == "rotate":
        t = _projection(case, g, case["B"] * case["Lq"])
        first = torch.randint(0, max(1, case["n_pos"] - case["Lq"]), (case["B"], 1), generator=g, device="cuda")
        t["positions"] = (first + torch.arange(case["Lq"], device="cuda")).int().contiguous()
        return t
    if kind == "append":
        old, new = _dealt(case)
        T = case["T"] + case["pad"]
        t = _projection(case, g, T)
        t.update(_pages(case, g, [a + b for a, b in zip(old, new)], 3, True))
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        t["cu"] = torch.tensor(cu, dtype=I32, device="cuda")
        t["seq_len"] = torch.tensor(old, dtype=I32, device="cuda")
        base = max(0, case["n_pos"] - 20000) // 2         # the user's tokens follow a fixed context
        pos = [base + a + j for a, b in zip(old, new) for j in range(b)] + [0] * case["pad"]
        t["positions"] = torch.tensor(pos, device="cuda").clamp(max=case["n_pos"] - 1).int()
        return t
    B, H, L = case["B"], case["H"], case["L"]
    if kind == "quantize":
        level = torch.exp(0.5 * torch.randn(2, B, H, 1, 1, generator=g, device="cuda"))      # heads differ in size
        t = dict(K=(level[0] * torch.randn(B, H, L, D, generator=g, device="cuda")).half(),
                 V=(level[1] * torch.randn(B, H, L, D, generator=g, device="cuda")).half(), perm=None)
        if case["perm"]:
            t["perm"] = torch.rand(B, H, L, generator=g, device="cuda").argsort(2).int()
        return t
    G, C = case["G"], case["C"]
    user = torch.randint(case["user"] // 2, case["user"] + 1, (B,), generator=g, device="cuda").int()
    user[0] = case["user"]
    t = _pages(case, g, [case["user"]] * B, 2)
    t.update(seq_len=user, q=(1.5 * torch.randn(B, H * G, 1, D, generator=g, device="cuda")).half())
    if not C:
        return t
    share = torch.tensor(_shares(case), device="cuda")
    R = share.numel()
    cuts = torch.randint(0, L + 1, (H, C - 1), generator=g, device="cuda").sort(1).values
    ends = torch.cat([cuts, torch.full((H, 1), L, device="cuda")], 1)
    first = torch.cat([torch.zeros(H, 1, dtype=ends.dtype, device="cuda"), cuts], 1)
    size = ends - first                                                                       # of exponential spread, zero among them
    head = torch.arange(R, device="cuda") // (1 if case["one_set"] else G) % H
    rank = torch.rand(R, C, generator=g, device="cuda").argsort(1).argsort(1)
    keep = (rank < (share * C).round().unsqueeze(1)) & (size[head] > 0)
    order = (~keep).int().sort(dim=1, stable=True).indices
    n = keep.sum(1)
    listed_ = torch.arange(C, device="cuda") < n.unsqueeze(1)
    ranges = torch.stack([torch.where(listed_, a[head].gather(1, order), 0) for a in (first, size)], 2).int()
    n_keys = ranges[:, :, 1].sum(1).int()
    t["most"] = int(n_keys.max())                                                             # (for the plain form's buffers)
    t.update(ranges=ranges.contiguous(), n_ranges=n.int(), n_keys=n_keys,
             K8=(64 * torch.randn(H, L, D, generator=g, device="cuda")).clamp(-448, 448).to(F8),
             V8=(64 * torch.randn(H, L, D, generator=g, device="cuda")).clamp(-448, 448).to(F8),
             ks=torch.exp2(torch.randint(-7, -5, (H, -(-L // BLOCK)), generator=g, device="cuda").float()),
             vs=torch.exp2(torch.randint(-7, -5, (H, -(-L // BLOCK)), generator=g, device="cuda").float()))
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    s = dict(case=case, t=t)
    e = lambda *sh, dtype=F16: torch.empty(*sh, dtype=dtype, device="cuda")  # noqa: E731
    kind, B, H = case["kind"], case["B"], case["H"]
    if kind == "rotate":
        Lq = case["Lq"]
        s.update(q=e(B, H * case["G"], Lq, D), k=e(B, H, Lq, D), v=e(B, H, Lq, D))
    elif kind == "append":
        s.update(q=torch.zeros(case["T"] + case["pad"], H * case["G"], D, dtype=F16, device="cuda"))
    elif kind == "quantize":
        L, n = case["L"], -(-case["L"] // BLOCK)
        s.update(K8=e(B, H, L, D, dtype=F8), V8=e(B, H, L, D, dtype=F8), ks=e(B, H, n, dtype=F32), vs=e(B, H, n, dtype=F32))
    else:
        s.update(out=e(B, H * case["G"], 1, D), lse=e(B, H * case["G"], 1, dtype=F32))
    if own:
        _plan(s)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# The framework's calls.
# ---------------------------------------------------------------------------------------------------------------------
def _plan(s):
    """What a program sets up once: the shape, the rotation's and the cache's descriptions, the workspace."""
    from paper_2411_09688_amd import binding as sq
    case, t = s["case"], s["t"]
    kind, B, H, G = case["kind"], case["B"], case["H"], case.get("G", 1)
    s["sq"] = sq
    if kind in ("rotate", "append"):
        s["rot"] = sq.make_rotary(t["table"], interleaved=t["adjacent"], q_weight=t["w_q"], k_weight=t["w_k"], eps=EPS)
    if kind in ("append", "attend"):
        s["cache"] = sq.make_cache(t["cK"], t["cV"], t["cks"], t["cvs"], t["pages"])
    if kind == "rotate":
        s["shape"] = sq.make_shape(B, H, 1, 1, case["Lq"], 0, SM_SCALE)
    elif kind == "append":
        s["shape"] = sq.make_shape(B, H, 1, 1, 1, 0, SM_SCALE)
        s["cu"] = None if case["T"] == B and not case["pad"] else t["cu"]
    elif kind == "quantize":
        s["shape"] = sq.make_shape(B, H, case["L"], 1, 1, 0, SM_SCALE)
    else:
        s["shape"] = sq.make_shape(B, H, case["L"], max(1, case["C"]), G, 0, SM_SCALE)
        s["ws"] = sq.workspace(s["shape"], sq.SQ_CALL_ATTN_DECODE_Q8, "cuda:0")


def _own(s):
    sq, case, t = s["sq"], s["case"], s["t"]
    kind = case["kind"]
    if kind == "rotate":
        sq.sq_head_norm_rotate(s["shape"], case["G"], s["rot"], t["positions"], t["q"], t["k"], t["v"], s["q"], s["k"], s["v"])
        return dict(q=s["q"], k=s["k"], v=s["v"])
    if kind == "append":
        sq.sq_cache_append(s["shape"], case["G"], s["rot"], s["cache"], t["seq_len"], t["positions"], t["q"], t["k"], t["v"], s["q"], s["cu"])
        return dict(q=s["q"], K8=t["cK"], V8=t["cV"], k_scale=t["cks"], v_scale=t["cvs"])
    if kind == "quantize":
        sq.sq_kv_quantize(s["shape"], t["K"], t["V"], t["perm"], s["K8"], s["V8"], s["ks"], s["vs"])
        return dict(K8=s["K8"], V8=s["V8"], k_scale=s["ks"], v_scale=s["vs"])
    sq.sq_sparse_attn_decode_q8(s["shape"], case["one_set"], t["q"], t.get("K8"), t.get("V8"), t.get("ks"), t.get("vs"), t.get("ranges"),
                                t.get("n_ranges"), t.get("n_keys"), s["cache"], t["seq_len"], s["out"], s["lse"], s["ws"])
    return dict(out=s["out"], lse=s["lse"])


# ---------------------------------------------------------------------------------------------------------------------
# Plain forms.
# ---------------------------------------------------------------------------------------------------------------------
def _normed_rotated(x, w, table, positions, adjacent, dtype):
    """x f16 [T, heads, 128]: norm over a head's row, then the rotation by the token's position, in `dtype`."""
    x = x.to(dtype)
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.to(dtype)
    cs = table[positions.long()].to(dtype).unsqueeze(1)                                      # [T, 1, rot / 2, 2]
    rot = 2 * table.shape[1]
    c, s = cs[..., 0], cs[..., 1]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if adjacent else (x[..., :rot // 2], x[..., rot // 2:rot])
    y = (a * c - b * s, b * c + a * s)
    y = torch.stack(y, -1).flatten(-2) if adjacent else torch.cat(y, -1)
    return torch.cat([y, x[..., rot:]], -1)


def _rounded(x):
    """To the nearest value of e4m3, ties to even (x within +-448): in x's own type, so that nothing is rounded twice."""
    step = torch.exp2((torch.frexp(x).exponent - 4).clamp(min=-9).to(x.dtype))
    return torch.round(x / step) * step


def _exponent(amax):
    """The least e with amax <= 448 * 2^e, within the limits."""
    m, e = torch.frexp(amax / 448)
    return torch.where(amax > 0, e - (m == 0.5).int(), E_MIN).clamp(E_MIN, E_MAX)


def _append_plain(x, t, codes, scales, block, old_end, old, page, off, real):
    """Rounds the tokens x [T, H, 128] into their pages, with the pages' scales raised where they ask for it.

    page, off [T]: where each token goes (real: whether it does); block, old_end [B]: the page that holds a sequence's
    last tokens so far, and how many; old [B]: whether such a page is appended to."""
    pages, H, P, _ = codes.shape
    amax = torch.zeros(pages, H, dtype=x.dtype, device=x.device)
    amax.index_reduce_(0, page, torch.where(real.view(-1, 1), x.abs().amax(-1), 0), "amax")
    count = lambda at, what: torch.zeros(pages, 1, dtype=I32, device=x.device).index_add_(0, at, what.int().view(-1, 1))  # noqa: E731
    touched, had = count(page, real) > 0, count(block, old) > 0
    e_old = torch.frexp(scales).exponent - 1
    e = torch.where(touched, torch.where(had, torch.maximum(e_old, _exponent(amax)), _exponent(amax)), e_old)
    raw = codes.view(U8)
    # what the page holds of earlier tokens, rounded again where the scale was raised
    was = raw[block].view(F8).float()
    again = _rounded(was * torch.exp2((e_old - e)[block].float())[..., None, None])
    mine = (torch.arange(P, device=x.device) < old_end.view(-1, 1)) & old.view(-1, 1)
    raw[block] = torch.where(mine[:, None, :, None], again, was).to(F8).view(U8)
    scales.copy_(torch.exp2(e.float()))
    y = _rounded(x / torch.exp2(e[page].to(x.dtype)).unsqueeze(-1)).float().to(F8).view(U8)
    here = raw[page, :, off]
    raw[page, :, off] = torch.where(real.view(-1, 1, 1), y, here)


def _plain(s):
    case, t = s["case"], s["t"]
    kind, B, H = case["kind"], case["B"], case["H"]
    if kind == "rotate":
        lay = lambda y: y.view(B, case["Lq"], -1, D).transpose(1, 2)  # noqa: E731
        pos = t["positions"].reshape(-1)
        s["q"].copy_(lay(_normed_rotated(t["q"], t["w_q"], t["table"], pos, t["adjacent"], F32)))
        s["k"].copy_(lay(_normed_rotated(t["k"], t["w_k"], t["table"], pos, t["adjacent"], F32)))
        s["v"].copy_(t["v"].reshape(B, case["Lq"], H, D).transpose(1, 2))
        return dict(q=s["q"], k=s["k"], v=s["v"])
    if kind == "append":
        T, P = t["k"].shape[0], case["page"]
        i = torch.arange(T, device="cuda")
        real = i < t["cu"][-1]
        b = (torch.searchsorted(t["cu"], i.int(), right=True) - 1).clamp(max=B - 1)
        slot = torch.where(real, t["seq_len"][b] + i - t["cu"][b], 0)
        # rows behind the last sequence point at a page that nobody has, and change nothing there
        free = torch.ones(t["cK"].shape[0], dtype=I32, device="cuda").index_fill_(0, t["pages"].flatten().long(), 0).argmax()
        page = torch.where(real, t["pages"][b, (slot // P).long()].long(), free)
        off = (slot % P).long()
        last = (t["seq_len"] // P).clamp(max=t["pages"].shape[1] - 1).long()
        block = t["pages"].gather(1, last.view(-1, 1))[:, 0].long()
        old_end = t["seq_len"] % P
        old = (old_end > 0) & (t["cu"][1:] > t["cu"][:-1])
        k = _normed_rotated(t["k"], t["w_k"], t["table"], t["positions"], t["adjacent"], F64)     # (its codes are decided at borders)
        _append_plain(k, t, t["cK"], t["cks"], block, old_end, old, page, off, real)
        _append_plain(t["v"].float(), t, t["cV"], t["cvs"], block, old_end, old, page, off, real)
        q = _normed_rotated(t["q"], t["w_q"], t["table"], t["positions"], t["adjacent"], F32).half()
        s["q"].copy_(torch.where(real.view(-1, 1, 1), q, s["q"]))
        return dict(q=s["q"], K8=t["cK"], V8=t["cV"], k_scale=t["cks"], v_scale=t["cvs"])
    if kind == "quantize":
        _quantize_plain(t["K"], t["perm"], s["K8"], s["ks"])
        _quantize_plain(t["V"], t["perm"], s["V8"], s["vs"])
        return dict(K8=s["K8"], V8=s["V8"], k_scale=s["ks"], v_scale=s["vs"])
    return _attend_plain(s, t, case)


def _quantize_plain(X, perm, codes, scales):
    B, H, L, _ = X.shape
    n = scales.shape[2]
    if perm is not None:
        X = X.gather(2, perm.long().unsqueeze(-1).expand(B, H, L, D))
    X = torch.nn.functional.pad(X.float(), (0, 0, 0, n * BLOCK - L)).view(B, H, n, BLOCK, D)
    e = _exponent(X.abs().amax((3, 4)))
    scales.copy_(torch.exp2(e.float()))
    codes.copy_((X / scales[..., None, None]).view(B, H, n * BLOCK, D)[:, :, :L].to(F8))


def _attend_plain(s, t, case):
    B, H, G, P = (case[k] for k in ("B", "H", "G", "page"))
    g = G if case["one_set"] else 1
    R = B * H * G // g
    q = t["q"].view(R, g, D).float()
    row = torch.arange(R, device="cuda")
    head, seq = row // (G // g) % H, row // (H * G // g)
    # the paged cache
    pos = torch.arange(case["user"], device="cuda")
    page = t["pages"][seq][:, pos // P].long()
    at = (page, head.view(-1, 1), (pos % P).view(1, -1))
    K = [t["cK"].view(U8)[at].view(F8).float() * t["cks"][at[:2]].unsqueeze(-1)]
    V = [t["cV"].view(U8)[at].view(F8).float() * t["cvs"][at[:2]].unsqueeze(-1)]
    ok = [pos < t["seq_len"][seq].view(-1, 1)]
    if case["C"]:
        count = t["ranges"][:, :, 1].long()
        ends = count.cumsum(1)
        pos = torch.arange(t["most"], device="cuda").expand(R, -1).contiguous()
        j = torch.searchsorted(ends, pos, right=True).clamp(max=case["C"] - 1)
        key = (t["ranges"][:, :, 0].long().gather(1, j) + pos - (ends - count).gather(1, j)).clamp(0, case["L"] - 1)
        at = (head.view(-1, 1), key)
        K.append(t["K8"].view(U8)[at].view(F8).float() * t["ks"][at[0], key // BLOCK].unsqueeze(-1))
        V.append(t["V8"].view(U8)[at].view(F8).float() * t["vs"][at[0], key // BLOCK].unsqueeze(-1))
        ok.append(pos < t["n_keys"].view(-1, 1))
    x = [torch.matmul(k, q.transpose(1, 2).contiguous()) * SM_SCALE for k in K]                      # [R, keys, g]
    x = [torch.where(o.unsqueeze(-1), v, -math.inf) for v, o in zip(x, ok)]
    m = torch.stack([v.amax(1) for v in x if v.shape[1]]).amax(0).unsqueeze(1)
    m = torch.where(torch.isfinite(m), m, 0.0)                                                       # (a row without keys)
    p = [torch.exp(v - m) for v in x]
    l = sum(v.sum(1) for v in p)
    o = sum(torch.matmul(v.transpose(1, 2).contiguous(), w) for v, w in zip(p, V))                   # [R, g, 128]
    s["out"].copy_(torch.where(l.unsqueeze(-1) > 0, o / l.unsqueeze(-1), 0.0).view(B, H * G, 1, D))
    s["lse"].copy_((m[:, 0] + torch.log(l)).view(B, H * G, 1))
    return dict(out=s["out"], lse=s["lse"])


def run(s):
    if own:
        return _own(s)
    return _plain(s)


def work(case):
    """Every input read once, every output written once; of the fixed context the keys that some row of a head keeps."""
    kind, B, H = case["kind"], case["B"], case["H"]
    G = case.get("G", 1)
    if kind in ("rotate", "append"):
        T = B * case["Lq"] if kind == "rotate" else case["T"]
        turned, out = (H * G + H) * T, 2 * D if kind == "rotate" else D
        bytes_ = T * (H * G * 4 * D + 2 * H * (2 * D + out)) + T * (4 * case["rot"] + 4)
        return dict(bytes=bytes_, flops=turned * (3.0 * case["rot"] + 4.0 * D * case["norm"]))
    if kind == "quantize":
        rows = B * H * case["L"]
        return dict(bytes=rows * (6 * D + 4 * case["perm"]) + 2 * B * H * (-(-case["L"] // BLOCK)) * 4, flops=4.0 * rows * D)
    per = 1 if case["one_set"] else G                      # rows of a (sequence, head)
    user = case["user"] * (0.75 * (B - 1) + 1) / B         # the mean length
    bytes_ = B * H * user * 2 * D + B * H * G * (4 * D + 4)
    flops = 4.0 * D * B * H * G * user
    if case["C"]:
        share = _shares(case)
        for h in range(H):
            rest = 1.0
            for b in range(B):
                for f in share[(b * H + h) * per:(b * H + h + 1) * per]:
                    rest *= 1.0 - f
            bytes_ += (1.0 - rest) * case["L"] * (2 * D + 8 / BLOCK)
        bytes_ += sum(share) * case["C"] * 8 + 8 * len(share)
        flops += 4.0 * D * case["L"] * sum(share) * (G if case["one_set"] else 1)
    return dict(bytes=bytes_, flops=flops)


# ---------------------------------------------------------------------------------------------------------------------
# The same in 64 bits, from the definitions, one sequence or head after the other.
# ---------------------------------------------------------------------------------------------------------------------
def _grid():
    """All finite values of e4m3 that are not negative, ascending: 8 of them per power of two."""
    small = torch.arange(8, dtype=F64, device="cuda") / 512
    return torch.cat([small] + [(1 + torch.arange(8, dtype=F64, device="cuda") / 8) * 2.0 ** e for e in range(-6, 9)])[:127]


def _nearest(x):
    """The value of the grid next to x; half way between two, the one of the even place."""
    grid = _grid()
    a = x.abs()
    i = torch.searchsorted(grid, a.contiguous(), right=True).sub(1).clamp(0, 125)
    lo, hi = grid[i], grid[i + 1]
    up = (a - lo > hi - a) | ((a - lo == hi - a) & (i % 2 == 1))
    return torch.where(up, hi, lo) * x.sign()


def _scale64(amax):
    """Powers of two tried from small to large: the first that holds amax within 448 times itself."""
    tried = 2.0 ** torch.arange(E_MIN, E_MAX + 1, dtype=F64, device="cuda")
    return tried[torch.searchsorted(448 * tried, amax.contiguous()).clamp(max=len(tried) - 1)]


def _turned64(x, w, t, positions):
    x = x.double()
    if w is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS) * w.double()
    y = x.clone()
    half = t["table"].shape[1]
    i = torch.arange(half, device="cuda")
    one, two = (2 * i, 2 * i + 1) if t["adjacent"] else (i, i + half)
    z = torch.complex(x[..., one], x[..., two]) * torch.view_as_complex(t["table"][positions.long()].double()).unsqueeze(1)
    y[..., one], y[..., two] = z.real, z.imag
    return y


def exact(case, seed):
    t = _inputs(case, seed)
    kind, B, H = case["kind"], case["B"], case["H"]
    if kind == "rotate":
        pos = t["positions"].flatten()
        lay = lambda y: y.view(B, case["Lq"], -1, D).permute(0, 2, 1, 3).contiguous()  # noqa: E731
        return dict(q=lay(_turned64(t["q"], t["w_q"], t, pos)), k=lay(_turned64(t["k"], t["w_k"], t, pos)), v=lay(t["v"].double().reshape(-1, H, D)))
    if kind == "append":
        old, new = _dealt(case)
        P = case["page"]
        q = _turned64(t["q"], t["w_q"], t, t["positions"])
        q[case["T"]:] = 0
        found = [q]
        table = t["pages"].cpu()
        for x, codes, scales in ((_turned64(t["k"], t["w_k"], t, t["positions"]), t["cK"], t["cks"]), (t["v"].double(), t["cV"], t["cvs"])):
            codes, scales = codes.double(), scales.double()
            at = 0
            for b in range(B):
                done = 0
                while done < new[b]:
                    slot = old[b] + done
                    n, o, page = min(P - slot % P, new[b] - done), slot % P, int(table[b, slot // P])
                    y = x[at + done:at + done + n].transpose(0, 1)                       # [H, n, 128]
                    sc = _scale64(y.abs().amax((1, 2)))
                    if o:
                        sc = torch.maximum(sc, scales[page])
                        codes[page, :, :o] = _nearest(codes[page, :, :o] * (scales[page] / sc).view(H, 1, 1))
                    codes[page, :, o:o + n] = _nearest(y / sc.view(H, 1, 1))
                    scales[page] = sc
                    done += n
                at += new[b]
            found += [codes, scales]
        return dict(q=found[0], K8=found[1], k_scale=found[2], V8=found[3], v_scale=found[4])
    if kind == "quantize":
        n = -(-case["L"] // BLOCK)
        out = {k: torch.empty(B, H, case["L"], D, dtype=F64, device="cuda") for k in ("K8", "V8")}
        out.update({k: torch.empty(B, H, n, dtype=F64, device="cuda") for k in ("k_scale", "v_scale")})
        for b in range(B):
            for h in range(H):
                for x, codes, scales in ((t["K"], "K8", "k_scale"), (t["V"], "V8", "v_scale")):
                    x = x[b, h].double() if t["perm"] is None else x[b, h].double()[t["perm"][b, h].long()]
                    row = x.abs().amax(1)
                    block = torch.arange(case["L"], device="cuda") // BLOCK
                    sc = _scale64(torch.zeros(n, dtype=F64, device="cuda").index_reduce_(0, block, row, "amax"))
                    out[scales][b, h] = sc
                    out[codes][b, h] = _nearest(x / sc[block].unsqueeze(1))
        return out
    G, P = case["G"], case["page"]
    per = 1 if case["one_set"] else G
    out = torch.empty(B, H * G, 1, D, dtype=F64, device="cuda")
    lse = torch.empty(B, H * G, 1, dtype=F64, device="cuda")
    lengths = t["seq_len"].tolist()
    for h in range(H):
        if case["C"]:
            block = torch.arange(case["L"], device="cuda") // BLOCK
            Kf, Vf = (t[a][h].double() * t[c][h].double()[block].unsqueeze(1) for a, c in (("K8", "ks"), ("V8", "vs")))
        for b in range(B):
            ids = t["pages"][b, :-(-lengths[b] // P)].long()
            Ku, Vu = ((t[a].view(U8)[ids, h].view(F8).double() * t[c][ids, h].double().view(-1, 1, 1)).reshape(-1, D)[:lengths[b]]
                      for a, c in (("cK", "cks"), ("cV", "cvs")))
            for i in range(per):
                r = (b * H + h) * per + i
                k, v = Ku, Vu
                if case["C"]:
                    first, count = t["ranges"][r, :, 0].long(), t["ranges"][r, :, 1].long()
                    mark = torch.zeros(case["L"] + 1, dtype=torch.long, device="cuda")
                    mark.index_add_(0, first, (count > 0).long()).index_add_(0, first + count, -(count > 0).long())
                    kept = mark.cumsum(0)[:-1] > 0
                    k, v = torch.cat([Kf[kept], k]), torch.cat([Vf[kept], v])
                heads = slice(h * G + i, h * G + i + 1) if per > 1 or G == 1 else slice(h * G, h * G + G)
                x = t["q"][b, heads, 0].double() @ k.T.contiguous() * SM_SCALE
                z = torch.logsumexp(x, 1, keepdim=True)
                out[b, heads, 0] = torch.exp(x - z) @ v
                lse[b, heads, 0] = z[:, 0]
    return dict(out=out, lse=lse)
