"""Linear attention's results held to their bounds head by head and, within a head, block by block of nodes, with the first and last
nodes on their own: in one norm over everything a head that never forgets hides what is wrong with one that forgets at once, and the middle
of a row its ends."""
import torch
from attention_util import linear_ref
from seq_util import FP32, ROUND, d64


def blocks(length):
    """Borders: each of the first and last two nodes, then 4, 8, 16 and so on of them, and every 32."""
    ends = [0, 1, 2, 4, 8, 16]
    return sorted({min(max(x, 0), length) for x in ends + [length - e for e in ends] + list(range(32, length, 32))})


def check_blocks(name, got, want, terms):
    """(batch, length, heads, features) each; terms: the same sums of their terms' sizes.

    The bound of a block's error, 2-norms: two half steps of the type and 1e-5 of the wanted block's own size, as everywhere, and 2^-22 of
    its terms': a sum of 32-bit products may cancel, and its rounding is then some 0.3 * 2^-24 of the terms (partial sums of random signs
    that each are rounded), of which this is more than ten times."""
    e, w, t = d64(got) - want, want, terms
    for lo, hi in zip(blocks(got.shape[1])[:-1], blocks(got.shape[1])[1:]):
        norm = [torch.linalg.vector_norm(x[:, lo:hi], dim=(1, 3)) for x in (e, w, t)]              # (batch, heads)
        lim = (2 * ROUND[got.dtype] + FP32) * norm[1] + 2.0 ** -22 * norm[2]
        assert bool((norm[0] <= lim).all()), "%s, nodes %d to %d: errors %s, bounds %s" % (name, lo, hi, norm[0].tolist(), lim.tolist())


def check_states(name, got, want, terms):
    """(batch, heads, dk, dv), head by head: fp32's bound whatever the arrays' type."""
    norm = [torch.linalg.vector_norm(x, dim=(2, 3)) for x in (d64(got) - want, want, terms)]
    assert bool((norm[0] <= FP32 * norm[1] + 2.0 ** -22 * norm[2]).all()), "%s: errors %s of %s" % (name, norm[0].tolist(), norm[1].tolist())


def wanted(q, k, v, ld, scale, s, go, gs):
    """[o, gq, gk, gv], [last state, its start's gradient or None] in 64 bits."""
    leaves = [t.requires_grad_(True) for t in (d64(q), d64(k), d64(v))]
    start = None if s is None else d64(s).requires_grad_(True)
    o, last = linear_ref(*leaves, d64(ld), scale, start)
    loss = (o * d64(go)).sum() + (0.0 if gs is None else (last * d64(gs)).sum())
    grads = torch.autograd.grad(loss, leaves + ([] if s is None else [start]), allow_unused=True)
    return [o.detach(), *grads[:3]], [last.detach(), grads[3] if s is not None else None]


def check_all(q, k, v, ld, scale, s, go, gs):
    """Both passes of linear attention against the 64-bit form."""
    from paper_2607_18020_b200 import sequence as Q
    o, last = Q.linear_attention_fwd(q, k, v, ld, scale, s)
    g = Q.linear_attention_bwd(go, q, k, v, ld, scale, s, gs)
    sizes = [None if t is None else t.abs() for t in (s, go, gs)]
    want, states = wanted(q, k, v, ld, scale, s, go, gs)
    terms, state_terms = wanted(q.abs(), k.abs(), v.abs(), ld, abs(scale), *sizes)
    for name, x, w, t in zip(("o", "gq", "gk", "gv"), (o, g.q, g.k, g.v), want, terms):
        check_blocks(name, x, w, t)
    for name, x, w, t in zip(("state", "gstate"), (last, g.state), states, state_terms):
        if x is not None:
            check_states(name, x, w, t)
