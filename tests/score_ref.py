"""Float64 definitions of the scores and losses of rows of logits, and bounds of what float32 sums may be off.

Bounds.  u = 2^-24.  An exponent a = (x - m) log2(e) / t takes three roundings (the difference, the factor, the
product) and a hardware exponential one unit in the last place (2 u), so exp a is off by at most
(3 |a| ln2 + 2) u of itself (|a| ln2 is |x - m| / t).  Sums of C positive numbers run in chains of at most
L = min(C, 128) + C / 1024 + 32 additions (registers of a lane, then lanes and waves, then passes over long rows):
L u of the sum.  So log s is off by ds = (L + 2 + 3 A) u with A = sum p |x - m| / t, and the hardware logarithm by
2 u |log s| more.
"""
import torch

U = 2.0 ** -24
INF = float("inf")
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}  # below: rounded in steps of it


def chain(C):
    return min(C, 128) + C / 1024 + 32


class Rows:
    """What the rows of logits x [T, C] come to at one temperature, in float64."""

    def __init__(self, x, temperature):
        self.x, self.t = x.double(), float(temperature)
        m = self.x.amax(1, keepdim=True)
        self.m = torch.where(m == -INF, torch.zeros_like(m), m)
        self.a = (self.x - self.m) / self.t
        e = self.a.exp()
        self.s = e.sum(1, keepdim=True)
        self.log_s = self.s.log()
        self.empty = self.s == 0
        self.p = torch.where(self.empty, torch.zeros_like(e), e / self.s)
        self.size = torch.where(self.a > -INF, self.a.abs(), torch.zeros_like(self.a))
        self.A = (self.p * self.size).sum(1, keepdim=True)
        self.A2 = (self.p * self.size ** 2).sum(1, keepdim=True)
        self.logp = torch.where(self.empty, torch.full_like(self.a, -INF), self.a - self.log_s)
        self.entropy = torch.where(self.empty, torch.zeros_like(self.s), self.log_s + self.A)
        self.lse = self.m / self.t + self.log_s
        C = x.shape[1]
        self.L = chain(C)
        self.ds = (self.L + 2 + 3 * self.A) * U + 2 * U * self.log_s.abs()

    def logp_off(self):
        return U * (3 * self.size + 4 * self.logp.abs()) + self.ds

    def lse_off(self):
        return self.ds + U * (2 * (self.m / self.t).abs() + 3 * self.log_s.abs() + self.lse.abs())

    def entropy_off(self):
        return self.ds * (1 + self.A) + U * (3 * self.A2 + (self.L + 7) * self.A + 3 * self.entropy.abs())

    def p_off(self):
        return self.p * (self.ds + U * (3 * self.size + 8)) + 2.0 ** -126


def pick(values, index, otherwise):
    """values[t, index[t]] of rows, `otherwise` where the index is outside."""
    inside = (index >= 0) & (index < values.shape[1])
    got = values.gather(1, index.clamp(0, values.shape[1] - 1).long()[:, None])[:, 0]
    return torch.where(inside, got, torch.full_like(got, otherwise))


def top(x, k):
    """Index of the k largest, equal ones by rising index, -1 where none above -inf is left; NaN is none."""
    y = torch.where(x.double().isnan(), torch.full_like(x.double(), -INF), x.double())
    value, at = torch.sort(y, dim=1, descending=True, stable=True)
    value, at = value[:, :k], at[:, :k]
    at = torch.where(value > -INF, at, torch.full_like(at, -1))
    if at.shape[1] < k:
        at = torch.cat([at, at.new_full((len(at), k - at.shape[1]), -1)], 1)
    return at.to(torch.int32)


def dense(index, value, C):
    """[T, C]: the entries of a row at their classes, added up."""
    inside = (index >= 0) & (index < C)
    full = torch.zeros(len(index), C, dtype=torch.float64, device=index.device)
    return full.scatter_add_(1, index.clamp(0, C - 1).long(), torch.where(inside, value.double(), torch.zeros_like(value.double())))


def rounded(off, exact, dtype):
    """The bound after rounding to the type."""
    return off + HALF_STEP[dtype] * (exact.abs() + off) + LEAST[dtype]


def backward(x, temperature, label=None, g_logp=None, g_lse=None, g_entropy=None, index=None, g_top=None):
    """The gradient, and how far float32 arithmetic may be off it (before the type's rounding)."""
    r = Rows(x, temperature)
    T, C = x.shape
    zero = torch.zeros(T, 1, dtype=torch.float64, device=x.device)
    point, size, k = torch.zeros(T, C, dtype=torch.float64, device=x.device), zero.clone(), 0
    for i, g in ((None if label is None else label[:, None], None if g_logp is None else g_logp[:, None]), (index, g_top)):
        if i is None or g is None:
            continue
        point += dense(i, g, C)
        size += (g.double().abs() * ((i >= 0) & (i < C))).sum(1, keepdim=True)
        k += i.shape[1]
    mass = point.sum(1, keepdim=True)
    gl = zero if g_lse is None else g_lse.double()[:, None]
    ge = zero if g_entropy is None else g_entropy.double()[:, None]
    surprise = torch.where(r.p > 0, r.a + r.A, torch.zeros_like(r.a))  # log p + H = a - mean of a
    d = point + r.p * (gl - mass - ge * surprise)
    off = r.p_off() * (size + gl.abs() + ge.abs() * (r.size + r.A))
    off += r.p * ((k + 6) * U * (size + gl.abs()) + ge.abs() * (6 * U * (r.size + r.A) + r.entropy_off() + 3 * U * r.size))
    off += (k + 6) * U * point.abs()
    off += U * dense(index, g_top.abs(), C) * k if index is not None and g_top is not None else 0.0
    d = torch.where(r.empty, torch.zeros_like(d), d) / r.t
    nothing = (mass == 0) & (gl == 0) & (ge == 0) & (point == 0).all(1, keepdim=True)
    return torch.where(nothing, torch.zeros_like(d), d), off / r.t


def distill(x, teacher, index, label, weight, hard, soft, temperature):
    """ce, kl, gradient, and the bounds of each (the gradient's before the type's rounding)."""
    T, C = x.shape
    cold, hot = Rows(x, 1.0), Rows(x, temperature)
    some_label = torch.zeros(T, 1, dtype=torch.bool, device=x.device)
    hit = torch.zeros(T, C, dtype=torch.float64, device=x.device)
    ce = ce_off = torch.zeros(T, dtype=torch.float64, device=x.device)
    if label is not None:
        some_label = ((label >= 0) & (label < C))[:, None]
        hit = dense(label[:, None], torch.ones(T, 1, device=x.device), C)
        ce, ce_off = -pick(cold.logp, label, 0.0), pick(cold.logp_off(), label, 0.0)
    inside = (index >= 0) & (index < C)
    t = torch.where(inside, teacher.double(), torch.full_like(teacher.double(), -INF))
    tr = Rows(t, temperature) if t.shape[1] else None
    kl = kl_off = torch.zeros(T, dtype=torch.float64, device=x.device)
    q = torch.zeros_like(t)
    some = torch.zeros(T, 1, dtype=torch.bool, device=x.device)
    q_off = torch.zeros_like(t)
    if tr is not None:
        q, some, q_off = tr.p, ~tr.empty, tr.p_off()
        at = index.clamp(0, C - 1).long()
        logp = hot.logp.gather(1, at)
        terms = torch.where(q > 0, q * (tr.logp - logp), torch.zeros_like(q))
        kl = torch.where(some[:, 0], terms.sum(1), kl)
        # each term's factors, the sum's chain, and both logarithms
        gap = torch.where(q > 0, tr.size + torch.where(logp > -INF, hot.size.gather(1, at), torch.zeros_like(q)), torch.zeros_like(q))
        kl_off = ((q * gap).sum(1) * (chain(t.shape[1]) + 8) * U + (q_off * gap).sum(1) + 4 * U * kl.abs() +
                  (tr.ds + hot.ds)[:, 0] + 4 * U * (tr.log_s.abs() + hot.log_s.abs())[:, 0])
    w = torch.ones(T, dtype=torch.float64, device=x.device) if weight is None else weight.double()
    full, full_off = dense(index, q, C), dense(index, q_off + (t.shape[1] + 4) * U * q, C)
    grad = hard * (cold.p * some_label - hit) + soft / temperature * (hot.p * some - full)
    off = abs(hard) * (cold.p_off() + 8 * U * (cold.p + hit)) + abs(soft) / temperature * (
        hot.p_off() + full_off + 8 * U * (hot.p + full))
    grad = torch.where(cold.empty, torch.zeros_like(grad), grad) * w[:, None]
    return ce, ce_off, kl, kl_off, grad, off * w.abs()[:, None]


def near(got, exact, off, what=""):
    """Every value within its bound; infinities and NaN in the same places."""
    got = got.double()
    assert got.shape == exact.shape, (what, got.shape, exact.shape)
    fine = exact.isfinite()
    assert torch.equal(fine, got.isfinite()), (what, "finite in other places")
    assert torch.equal(exact.isnan(), got.isnan()), (what, "NaN in other places")
    odd = ~fine & ~exact.isnan()
    assert torch.equal(exact[odd], got[odd]), (what, "other infinities")
    far = ((got - exact).abs() > off) & fine
    if bool(far.any()):
        i = int((((got - exact).abs() / off).masked_fill(~far, 0)).argmax())
        i = tuple(int(v) for v in torch.unravel_index(torch.tensor(i), exact.shape))
        raise AssertionError((what, i, float(got[i]), float(exact[i]), float(off[i])))
