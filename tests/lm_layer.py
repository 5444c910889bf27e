"""A residual block of a language model out of the 8-bit layer's operators, once for any set of them (test infrastructure)."""
import numpy as np

import lm_plain as plain

EPS, RES, BRANCH, P = 1e-5, 0.9, 0.6, 0.25


def block(o, x):
    """Forward and backward of  norm - product - drop-out - product - norm, gate, drop-out, sum, norm.  x: the inputs by name; o: the
    operators.  Codes come as a pair (over the rows, over the columns).  Returns outputs and gradients by name."""
    _, y1, st1 = o.norm(x["res"], None, None, None, x["w_in"])
    a, w1, w2 = o.codes(y1), o.weight(x["w1"]), o.weight(x["w2"])
    z = o.product(a[0], w1[1])
    b = o.codes(o.drop(z))
    h = o.product(b[0], w2[1])
    outer = (x["w_post"], x["gate"], x["w_pre"])
    res2, y2, st2 = o.norm(x["res"], h, *outer)
    dres, dh, dgate, dw_post, dw_pre = o.norm_bwd(x["dy"], x["dres"], res2, h, st2, *outer)
    g = o.gradient(dh)
    f = o.gradient(o.drop(o.product(g[0], w2[0])))
    dres, _, _, _, dw_in = o.norm_bwd(o.product(f[0], w1[0]), dres, x["res"], None, st1, None, None, x["w_in"])
    return dict(res2=res2, y2=y2), dict(res=dres, w_in=dw_in, w1=o.product(a[1], f[1], True), w2=o.product(b[1], g[1], True), gate=dgate,
                                        w_post=dw_post, w_pre=dw_pre)


def inputs(T, D, N, groups, seed=0):
    g = np.random.default_rng(seed)
    n = g.standard_normal
    return dict(res=n((T, D)), w_in=1 + 0.3 * n(D), w1=n((D, N)) / np.sqrt(D), w2=n((N, D)) / np.sqrt(N), gate=0.5 + 0.5 * n((groups, D)),
                w_post=1 + 0.3 * n(D), w_pre=1 + 0.3 * n(D), dy=n((T, D)), dres=n((T, D)))


class Exact:
    """the operators in 64 bits, without the rounding to codes"""

    def keep(self, shape, seed):
        return plain.kept(int(np.prod(shape)), P, seed).reshape(shape)

    def norm(self, res, h, w_post, gate, w_pre):
        r, y, s1, s2 = plain.norm_fwd(res, h, w_post, gate, w_pre, EPS, RES, BRANCH, None if h is None else self.keep(h.shape, 5))
        return r, y, (s1, s2)

    def norm_bwd(self, dy, dres_out, r, h, st, w_post, gate, w_pre):
        scales = (1.0, 1.0, None) if h is None else (RES, BRANCH, self.keep(h.shape, 5))
        return plain.norm_bwd(dy, dres_out, r, h, *st, w_post, gate, w_pre, *scales)

    def codes(self, x):
        return x, x.T

    weight = gradient = codes

    def product(self, a, b, whole=False):
        return a @ b.T

    def drop(self, z):
        return plain.dropout(z, P, 6)
