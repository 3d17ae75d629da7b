"""Comparison of the attention calls with their fp64 definitions, element by element, and its bounds.

u is half a step of the operands' type (bf16 2^-8, fp32 2^-24): results are rounded to it once, and with bf16 so are the probabilities and
dS, operands of the matrix cores.  Everything else is fp32: a score of dim terms is off by (dim + 8) 2^-24 of the sum of its terms' sizes,
the argument of an exponential by 2^-23 of its parts, an exponential by 2^-22 of itself; a sum of n terms by (n + 8) 2^-24 of their sizes."""
import numpy as np

from oracle import attn_oracle as ao

from gpu_util import host

E = 2.0 ** -24


def half_step(kind):
    return 2.0 ** -8 if kind == "bf16" else E


def heads_of(x, heads):
    """[rows][heads * dim] -> [heads][rows][dim] fp64"""
    x = host(x).astype(np.float64)
    return x.reshape(x.shape[0], heads, -1).transpose(1, 0, 2)


def starts(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def within(got, ref, tol, what):
    assert np.isfinite(got).all(), f"{what}: not finite"
    bad = np.abs(got - ref) > tol
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.abs(got - ref)[bad].max():.3e} where {tol[bad].min():.3e} is allowed"


def near(got, ref, size, rest, what):
    """In the 2-norm: errors of `size` (the root of the summed squares of what is rounded) are roundings that do not depend on each other, each
    0.42 half steps in the mean; three times that is allowed, and `rest` of what is not."""
    err, room = np.linalg.norm(got - ref), 1.25 * np.linalg.norm(size) + np.linalg.norm(rest)
    assert err <= room, f"{what}: {err:.3e} in the 2-norm where {room:.3e} is allowed (result {np.linalg.norm(ref):.3e})"


def _spread(z_size, lse, dim):
    """relative error of a probability: the score, the arguments of the exponential, the exponential"""
    return 2 * (dim + 8) * E * z_size + 2 * E * 1.5 * (2 * z_size + np.abs(np.where(np.isfinite(lse), lse, 0.0))[:, None]) + 4 * 2 * E


def check_fwd(o, lse, q, k, v, qlens, klens, heads, kv, scale, causal, window, sinks, kind):
    u, dim = half_step(kind), q.shape[1] // heads
    Q, K, V, O = heads_of(q, heads), heads_of(k, kv), heads_of(v, kv), heads_of(o, heads)
    L = host(lse)
    qs, ks = starts(qlens), starts(klens)
    for s, (nq, nk) in enumerate(zip(qlens, klens)):
        if nq == 0:
            continue
        mask = ao.seen(nq, nk, causal, window, sinks)
        for h in range(heads):
            a, b = slice(qs[s], qs[s + 1]), slice(ks[s], ks[s + 1])
            x, y, z = Q[h, a], K[h * kv // heads, b], V[h * kv // heads, b]
            ref, rl, p = ao.attention_fwd(x, y, z, scale, mask)
            size = scale * (np.abs(x) @ np.abs(y).T)
            eta = np.where(mask, _spread(size, rl, dim), 0.0)
            parts = (p * (u + eta + eta.max(1, keepdims=True, initial=0.0) + (nk + 8) * E)) @ np.abs(z)
            within(O[h, a], ref, 1.01 * u * np.abs(ref) + 1.01 * parts + 1e-30, f"o of sequence {s} head {h}")
            if kind == "bf16":
                near(O[h, a], ref, u * np.sqrt(ref ** 2 + p ** 2 @ z ** 2), (p * (eta + eta.max(1, keepdims=True, initial=0.0) + (nk + 8) * E)) @ np.abs(z),
                     f"o of sequence {s} head {h}")
            empty = ~mask.any(1)
            assert (L[h, a][empty] == -np.inf).all() and (O[h, a][empty] == 0).all()
            within(L[h, a][~empty], rl[~empty], (eta.max(1, initial=0.0) + (nk + 8) * E + 4 * E * np.abs(np.where(empty, 0, rl)))[~empty],
                   f"lse of sequence {s} head {h}")


def check_bwd(dq, dk, dv, do, q, k, v, o, lse, qlens, klens, heads, kv, scale, causal, window, sinks, kind):
    u, dim, group = half_step(kind), q.shape[1] // heads, heads // kv
    Q, K, V, O, G = heads_of(q, heads), heads_of(k, kv), heads_of(v, kv), heads_of(o, heads), heads_of(do, heads)
    DQ, DK, DV = heads_of(dq, heads), heads_of(dk, kv), heads_of(dv, kv)
    qs, ks = starts(qlens), starts(klens)
    for s, (nq, nk) in enumerate(zip(qlens, klens)):
        mask = ao.seen(nq, nk, causal, window, sinks)
        a, b = slice(qs[s], qs[s + 1]), slice(ks[s], ks[s + 1])
        for g in range(kv):
            y, z = K[g, b], V[g, b]
            rk, rv, tk, tv, sk, sv, fk, fv = (np.zeros((nk, dim)) for _ in range(8))
            for h in range(g * group, (g + 1) * group):
                x, d, oo = Q[h, a], G[h, a], O[h, a]
                exact_o, rl, p = ao.attention_fwd(x, y, z, scale, mask)
                rq, one_k, one_v, ds = ao.attention_bwd(d, x, y, z, exact_o, p, scale)
                size = scale * (np.abs(x) @ np.abs(y).T)
                # P is formed from lse, which is off by as much as the forward's
                eta = np.where(mask, _spread(size, rl, dim), 0.0)
                eta = eta + eta.max(1, keepdims=True, initial=0.0) + (nk + 8) * E
                dp, delta = np.abs(d @ z.T), np.abs((d * exact_o).sum(1, keepdims=True))
                # fp32: do . o takes the o that the forward rounded.  bf16: what that lacks is put back, by sums of P in bf16: half steps of half steps
                size_o = (np.abs(d) * (np.abs(oo) + np.abs(exact_o))).sum(1, keepdims=True)
                inner = (dim + 8) * E * (np.abs(d) @ np.abs(z).T + size_o) + (2 * u * u * size_o if kind == "bf16" else 0.0)
                fine = p * (eta * (dp + delta) + inner + 4 * E * (dp + delta))
                err = fine + u * np.abs(ds)
                tq = scale * ((err + (nk + 8) * E * np.abs(ds)) @ np.abs(y))
                if nq:
                    within(DQ[h, a], rq, 1.01 * u * np.abs(rq) + 1.01 * tq + 1e-30, f"dq of sequence {s} head {h}")
                    if kind == "bf16":
                        near(DQ[h, a], rq, u * np.sqrt(rq ** 2 + scale ** 2 * ds ** 2 @ y ** 2), scale * ((fine + (nk + 8) * E * np.abs(ds)) @ np.abs(y)),
                             f"dq of sequence {s} head {h}")
                n = (nq * group + 8) * E
                tk += scale * ((err + n * np.abs(ds)).T @ np.abs(x))
                tv += (p * (u + eta + n)).T @ np.abs(d)
                sk += scale ** 2 * (ds ** 2).T @ x ** 2
                sv += (p ** 2).T @ d ** 2
                fk += scale * ((fine + n * np.abs(ds)).T @ np.abs(x))
                fv += (p * (eta + n)).T @ np.abs(d)
                rk += one_k
                rv += one_v
            if nk:
                within(DK[g, b], rk, 1.01 * u * np.abs(rk) + 1.01 * tk + 1e-30, f"dk of sequence {s} head {g}")
                within(DV[g, b], rv, 1.01 * u * np.abs(rv) + 1.01 * tv + 1e-30, f"dv of sequence {s} head {g}")
                if kind == "bf16":
                    near(DK[g, b], rk, u * np.sqrt(rk ** 2 + sk), fk, f"dk of sequence {s} head {g}")
                    near(DV[g, b], rv, u * np.sqrt(rv ** 2 + sv), fv, f"dv of sequence {s} head {g}")
