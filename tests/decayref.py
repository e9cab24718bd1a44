"""The linear attention with decays in fp64, row by row, on the CPU, with what its kernels
may be off by.

Every result is a sum of terms, and so is the same recurrence over the absolute values: the
tolerances are parts of that.  A term's weight a^n is off by n |log a| 2 U + 2 U of itself,
which times its e^(-n |log a|) is below 3 U of the largest there is; the sums over heads'
columns, over the rows of a chunk and from chunk to chunk add at most some 200 roundings one
after another on the way to a result: SUMS = 256 U.  With 16-bit inputs one factor of every
term of a row's result is rounded once more (the weight within a chunk, or the state): half
a step of the type; states themselves take 2^-21 at most from the splitting of 16-bit operands."""
import torch

from opref import F64, U, cpu64, half_step

SUMS = 256 * U


def chains(begin, end, reverse):
    return [list(range(b, e))[::-1 if reverse else 1] for b, e in zip(begin, end)]


def run(q, k, v, g, scale, heads, kv_heads, rows_of, state=None, do=None, dstate_last=None):
    """dict of results and of the sums of absolute values ("abs_" + name); ``rows_of``: each
    sequence's rows in order."""
    q, k, v, g, state, do, dstate_last = cpu64(q, k, v, g, state, do, dstate_last)
    R, H, G, S = q.shape[0], heads, kv_heads, len(rows_of)
    q = q.reshape(R, H, q.shape[1] // H)
    share = lambda m: m.reshape(R, G, m.shape[1] // G).repeat_interleave(H // G, 1)
    k, v = share(k), share(v)
    dk, dv = k.shape[2], v.shape[2]
    a = torch.exp(g)[:, None, None]
    new = lambda *s: torch.zeros(*s, dtype=F64)
    out = dict(o=new(R, H, dv), state_last=new(S, H, dk, dv))
    if do is not None:
        do = do.reshape(R, H, dv)
        out.update(dq=new(R, H, dk), dk=new(R, H, dk), dv=new(R, H, dv), dstate=new(S, H, dk, dv))
    out.update({"abs_" + n: torch.zeros_like(t) for n, t in list(out.items())})
    sizes = [("", lambda t: t)] + [("abs_", torch.abs)]
    for pre, f in sizes:
        fq, fk, fv, sc = f(q), f(k), f(v), (abs(scale) if pre else scale)
        fo = None if do is None else f(do)
        for s, rows in enumerate(rows_of):
            st = new(H, dk, dv) if state is None else f(state[s]).clone()
            for r in rows:
                st = a * st + fk[r][:, :, None] * fv[r][:, None, :]
                out[pre + "o"][r] = sc * (fq[r][:, None] @ st)[:, 0]
                if fo is not None:
                    out[pre + "dq"][r] = sc * (st @ fo[r][:, :, None])[:, :, 0]
            out[pre + "state_last"][s] = st
            if fo is None:
                continue
            d = new(H, dk, dv) if dstate_last is None else f(dstate_last[s]).clone()
            for i, r in enumerate(reversed(rows)):
                d = (a * d if i else d) + sc * fq[r][:, :, None] * fo[r][:, None, :]
                out[pre + "dk"][r] = (d @ fv[r][:, :, None])[:, :, 0]
                out[pre + "dv"][r] = (fk[r][:, None] @ d)[:, 0]
            out[pre + "dstate"][s] = a * d if rows else d
    flat = lambda t: t.reshape(R, -1)
    group = lambda t: flat(t.reshape(R, G, H // G, -1).sum(2))
    for n in list(out):
        name = n.replace("abs_", "")
        if name in ("o", "dq"):
            out[n] = flat(out[n])
        elif name in ("dk", "dv"):
            out[n] = group(out[n])
    return out


def tolerance(name, ref, dtype):
    """Before the rounding of a result to its type."""
    a = ref["abs_" + name]
    if dtype == torch.float32:
        return SUMS * a
    if name in ("state_last", "dstate"):
        return (SUMS + 2.0 ** -21) * a
    return (SUMS + 2.0 ** -21 + half_step(dtype)) * a
