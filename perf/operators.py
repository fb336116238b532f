"""The LM head in training and in four bits: cases that can be timed and compared.

  xent      dart_lmhead_xent_fwd_bwd: cross entropy of the LM head's inputs (tokens left out, label
            smoothing, z-loss) with its gradients; the logits are never kept
  eval      dart_lmhead_xent_fwd: the loss alone
  quant     dart_mxfp4_quantize and dart_mxfp4_dequantize: a matrix in blocks of 32 four-bit
            values with a power-of-two scale, and the values that it stands for
  product   dart_mxfp4_matmul: the logits of tokens under a head kept in four bits
  head4     dart_lmhead_mxfp4_tok_stats: log-probs, entropies and normalisers under such a head

Where `own` is false the same values come from elementary torch operations in float32.
"""

import math

import numpy as np
import torch

own = False


def listed():
    return [
        # a few tokens of a small model: launches and latency
        dict(name="xent_small", kind="xent", T=48, V=4000, d=512, left_out=0.25, smooth=0.0, z=0.0),
        # one episode's tokens under the 7B policy's head, prompts left out, smoothed targets
        dict(name="xent_episode", kind="xent", T=1000, V=152064, d=3584, left_out=0.3, smooth=0.1, z=0.0),
        # a step group's tokens under it, all of them learnt from, with a z-loss
        dict(name="xent_group", kind="xent", T=4096, V=152064, d=3584, left_out=0.0, smooth=0.0, z=1e-4),
        # held-out loss of a medium model with an odd vocabulary
        dict(name="eval_odd", kind="eval", T=2000, V=50257, d=2048, left_out=0.1, smooth=0.0, z=0.0),
        # the hidden states of a decoding batch, on their way into a four-bit product
        dict(name="quant_tokens", kind="quant", R=64, K=3584, dtype="bf16"),
        # rows that end inside a block, in float32
        dict(name="quant_ragged", kind="quant", R=5001, K=1001, dtype="f32"),
        # the 7B policy's head, handed to the rollout
        dict(name="quant_head", kind="quant", R=152064, K=3584, dtype="bf16"),
        # the next token's logits of one sequence
        dict(name="product_token", kind="product", M=1, N=152064, K=3584, out="bf16"),
        # those of a decoding batch of a small model, odd sizes, float32 logits
        dict(name="product_batch", kind="product", M=48, N=32003, K=2056, out="f32"),
        # the logits of a step group
        dict(name="product_group", kind="product", M=4096, N=152064, K=3584, out="bf16"),
        # one step's tokens scored under the rollout's head
        dict(name="head4_step", kind="head4", T=64, V=152064, d=3584, inv_temp=1.0),
        # a step group scored under it
        dict(name="head4_group", kind="head4", T=4096, V=152064, d=3584, inv_temp=1.25),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, evenly spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: one token to a step group, vocabularies from 1000 to 152064 and hidden sizes
    from 64 to 3584, odd ones among them."""
    kind = rng.choice(["xent", "xent", "eval", "quant", "product", "product", "head4"])
    V = _spread(rng, 1000, 152064)
    V = V if rng.random() < 0.5 else V // 64 * 64
    d = _spread(rng, 64, 3584) // 8 * 8
    c = dict(kind=kind)
    if kind in ("xent", "eval"):
        c.update(T=_spread(rng, 1, 4096), V=V, d=d, left_out=rng.choice([0.0, 0.2, 0.5, 0.8]),
                 smooth=rng.choice([0.0, 0.0, 0.05, 0.1]), z=rng.choice([0.0, 0.0, 1e-4, 1e-3]))
    elif kind == "quant":
        c.update(R=_spread(rng, 1, 152064), K=_spread(rng, 32, 3584), dtype=rng.choice(["bf16", "bf16", "f32"]))
        if rng.random() < 0.5:
            c["K"] = c["K"] // 32 * 32
    elif kind == "product":
        c.update(M=_spread(rng, 1, 4096), N=V, K=d, out=rng.choice(["bf16", "f32"]))
    else:
        c.update(T=_spread(rng, 1, 4096), V=V, d=d, inv_temp=rng.choice([1.0, 1.0, 0.8, 1.25]))
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------


def _kept(T, left_out):
    """Which of T tokens are learnt from: in each of up to eight episodes the first share is its prompt."""
    episode = -(-T // 8)
    return np.arange(T) % episode >= int(episode * left_out)


def _head(g, T, V, d, dev):
    """Hidden states, an LM-head weight and targets in bf16 and int32: logits of standard deviation 3,
    the target's raised by up to 16, so that its probability runs from next to nothing to most."""
    w = (torch.randn((V, d), generator=g, device=dev) * (3.0 / math.sqrt(d))).to(torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=g, device=dev, dtype=torch.int32)
    wy = w[y.long()].float()
    up = torch.rand((T, 1), generator=g, device=dev) * 16.0 / wy.square().sum(1, keepdim=True)
    h = (torch.randn((T, d), generator=g, device=dev) + up * wy).to(torch.bfloat16)
    return h, w, y


def _values(g, R, K, dev):
    """Rows of values whose size differs from row to row and, for one in a hundred, by far."""
    x = torch.randn((R, K), generator=g, device=dev)
    x *= torch.exp2(torch.randint(-6, 7, (R, 1), generator=g, device=dev).float())
    far = torch.rand((R, K), generator=g, device=dev) < 0.01
    return torch.where(far, x * 20.0, x)


def _inputs(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 1000003 + 17)
    kind = case["kind"]
    if kind == "quant":
        x = _values(g, case["R"], case["K"], dev)
        return dict(x=x.to(torch.bfloat16) if case["dtype"] == "bf16" else x)
    if kind == "product":
        h, w, _ = _head(g, case["M"], case["N"], case["K"], dev)
        return dict(h=h, w=w)
    h, w, y = _head(g, case["T"], case["V"], case["d"], dev)
    if kind != "head4":
        keep = torch.from_numpy(_kept(case["T"], case["left_out"])).to(dev)
        y = torch.where(keep, y, torch.full_like(y, -100))
    return dict(h=h, w=w, y=y)


def prepare(case, seed):
    state = dict(case=case, **_inputs(case, seed))
    if case["kind"] in ("product", "head4"):
        # the head in four bits is what a rollout keeps
        if own:
            import paper_2509_23866_amd as dart

            state["w"] = dart.dart_mxfp4_quantize(state["w"])
        else:
            state["w"] = _four_bits(state["w"].float()).to(torch.bfloat16)  # exact: 2 bits and a power of two
    return state


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------


def _four_bits(x):
    """The values that the rows of float32 x stand for in four bits: per block of 32 the largest power of
    two not above its largest size, divided by 4, times the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6."""
    R, K = x.shape
    b = torch.nn.functional.pad(x, (0, -K % 32)).view(R, -1, 32)
    _, e = torch.frexp(b.abs().amax(2, keepdim=True))
    e = torch.clamp(e - 3, min=-127)
    a = torch.ldexp(b, -e).abs()
    q = 0.5 * ((a > 0.25).float() + (a >= 0.75).float() + (a > 1.25).float() + (a >= 1.75).float())
    q = q + (a > 2.5).float() + (a >= 3.5).float() + 2.0 * (a > 5.0).float()
    return torch.copysign(torch.ldexp(q, e), b).view(R, -1)[:, :K]


def _log_softmax_parts(z, y):
    """(z of the target, normaliser) of rows of float32 logits."""
    m = z.amax(1, keepdim=True)
    lse = (m + (z - m).exp().sum(1, keepdim=True).log())[:, 0]
    return z.gather(1, y.long()[:, None])[:, 0], lse


def _plain_xent(s, grads):
    c, h, w, y = s["case"], s["h"].float(), s["w"].float(), s["y"]
    keep = y >= 0
    safe = torch.where(keep, y, torch.zeros_like(y))
    n = keep.sum(dtype=torch.int32)
    z = h @ w.t()
    zy, lse = _log_softmax_parts(z, safe)
    eps, lam, V = c["smooth"], c["z"], c["V"]
    # the difference of two numbers of the logits' size, next to 0 for a sure target
    tok = (lse.double() - (1.0 - eps) * zy.double() - (eps / V) * z.double().sum(1)
           + lam * lse.double().square())
    tok = torch.where(keep, tok, torch.zeros_like(tok))
    loss = tok.sum() / n.clamp(min=1)
    out = [loss.float().view(1), tok.float(), n.view(1)]
    if grads:
        dz = (z - lse[:, None]).exp() * (1.0 + 2.0 * lam * lse)[:, None] - eps / V
        dz.scatter_add_(1, safe.long()[:, None], torch.full_like(lse, eps - 1.0)[:, None])
        dz *= (keep / n.clamp(min=1))[:, None]
        out += [(dz @ w).to(torch.bfloat16), (dz.t() @ h).to(torch.bfloat16)]
    return out


def _plain_stats(s):
    c = s["case"]
    z = (_four_bits(s["h"].float()) @ s["w"].float().t()) * c["inv_temp"]
    zy, lse = _log_softmax_parts(z, s["y"])
    lp = z - lse[:, None]
    return [zy - lse, -(lp.exp() * lp).sum(1), lse]


def _plain(s):
    c = s["case"]
    if c["kind"] in ("xent", "eval"):
        return _plain_xent(s, c["kind"] == "xent")
    if c["kind"] == "quant":
        return _four_bits(s["x"].float()).to(s["x"].dtype)
    if c["kind"] == "product":
        z = _four_bits(s["h"].float()) @ s["w"].float().t()
        return z.to(torch.bfloat16) if c["out"] == "bf16" else z
    return _plain_stats(s)


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------


def _own(s):
    import paper_2509_23866_amd as dart

    c = s["case"]
    if c["kind"] == "xent":
        return list(dart.dart_lmhead_xent_fwd_bwd(s["h"], s["w"], s["y"], label_smoothing=c["smooth"],
                                                  z_loss=c["z"]))
    if c["kind"] == "eval":
        return list(dart.dart_lmhead_xent_fwd(s["h"], s["w"], s["y"], label_smoothing=c["smooth"],
                                              z_loss=c["z"]))
    if c["kind"] == "quant":
        return dart.dart_mxfp4_dequantize(dart.dart_mxfp4_quantize(s["x"]), dtype=s["x"].dtype)
    if c["kind"] == "product":
        return dart.dart_mxfp4_matmul(s["h"], s["w"],
                                      dtype=torch.bfloat16 if c["out"] == "bf16" else torch.float32)
    return list(dart.dart_lmhead_mxfp4_tok_stats(s["h"], s["w"], s["y"], inv_temp=c["inv_temp"]))


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and what it should give
# ---------------------------------------------------------------------------


def work(case):
    c = case
    if c["kind"] == "quant":
        size = 2 if c["dtype"] == "bf16" else 4
        # the matrix, its four-bit form, its values
        return {"bytes": c["R"] * (c["K"] * 2 * size + -(-c["K"] // 32) * 17), "flops": 0}
    if c["kind"] == "product":
        size = 2 if c["out"] == "bf16" else 4
        return {"bytes": c["M"] * c["K"] * 2 + c["N"] * (-(-c["K"] // 32) * 17) + c["M"] * c["N"] * size,
                "flops": 2 * c["M"] * c["N"] * c["K"]}
    T, V, d = c["T"], c["V"], c["d"]
    if c["kind"] == "head4":
        return {"bytes": T * d * 2 + V * (-(-d // 32) * 17) + T * 16, "flops": 2 * T * V * d}
    n = int(_kept(T, c["left_out"]).sum())
    read = n * d * 2 + V * d * 2 + T * 8
    if c["kind"] == "eval":
        return {"bytes": read, "flops": 2 * n * V * d}
    return {"bytes": read + T * d * 2 + V * d * 2, "flops": 6 * n * V * d}


def _exact_four_bits(x):
    """float64: each value to the one of the fifteen of its block's scale that is nearest, of two as near
    the one with an even code."""
    x = x.double()
    R, K = x.shape
    full = torch.zeros((R, -(-K // 32) * 32), dtype=torch.float64, device=x.device)
    full[:, :K] = x
    b = full.view(-1, 32)
    top = b.abs().max(1).values
    e = torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top))))
    e = torch.where(torch.exp2(e) > top, e - 1, e)  # a logarithm rounded up to the next whole number
    e = torch.where(torch.exp2(e + 1) <= top, e + 1, e)
    scale = torch.exp2(torch.where(top > 0, torch.clamp(e - 2, min=-127.0), torch.full_like(e, -127.0)))
    size = b.abs() / scale[:, None]
    best = torch.zeros_like(size)
    gap = size.clone()
    for value, even in ((0.5, False), (1.0, True), (1.5, False), (2.0, True), (3.0, False), (4.0, True),
                        (6.0, False)):
        off = (size - value).abs()
        nearer = (off <= gap) if even else (off < gap)
        best = torch.where(nearer, torch.full_like(best, value), best)
        gap = torch.where(nearer, off, gap)
    return (torch.sign(b) * best * scale[:, None]).view(R, -1)[:, :K]


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["kind"] == "quant":
        return _exact_four_bits(s["x"])
    w = s["w"]
    if c["kind"] in ("product", "head4"):
        w = torch.cat([_exact_four_bits(part) for part in w.split(8192)])
        logits = _exact_four_bits(s["h"]) @ w.t()
        if c["kind"] == "product":
            return logits
        lp = torch.log_softmax(logits * c["inv_temp"], 1)
        at = s["y"].long()[:, None]
        logp = lp.gather(1, at)[:, 0]
        lse = logits.gather(1, at)[:, 0] * c["inv_temp"] - logp
        return [logp, torch.special.entr(lp.exp_()).sum(1), lse]
    # rows that are learnt from only
    rows = torch.nonzero(s["y"] >= 0)[:, 0]
    N, V = rows.numel(), c["V"]
    h, w, y = s["h"][rows].double(), w.double(), s["y"][rows].long()
    logits = h @ w.t()
    lse = torch.logsumexp(logits, 1)
    want = torch.full_like(logits, c["smooth"] / V)  # the distribution to be learnt
    want[torch.arange(N, device=y.device), y] += 1.0 - c["smooth"]
    tok = torch.zeros(c["T"], dtype=torch.float64, device=y.device)
    tok[rows] = ((lse[:, None] - logits) * want).sum(1) + c["z"] * lse ** 2
    out = [tok.sum().view(1) / max(N, 1), tok, None]
    if c["kind"] == "xent":
        d_lse = 1.0 + 2.0 * c["z"] * lse
        dz = (torch.softmax(logits, 1) * d_lse[:, None] - want) / max(N, 1)
        dh = torch.zeros((c["T"], c["d"]), dtype=torch.float64, device=y.device)
        dh[rows] = dz @ w
        out += [dh, dz.t() @ h]
    return out
