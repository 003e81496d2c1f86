"""The experts' products (fl_moe_expert_*) against the formulas in 64 bits, and their refusals.

Tolerances are bounds, derived here once.  A sum of k products in fp32, in any order, each step off by at most one unit
in the last place (2^-23) of what has been summed: off by at most k 2^-23 sum |a b|.  A result rounded to bf16: half a
step, 2^-8 of the value; to an e4m3 block: 2^-4 of the value or half the smallest step, 2^-10 of the scale.
Inputs of bf16 or e4m3 are exact in 64 bits.

The matrix instruction for e4m3 adds the products of eight neighbours of the contraction after it has cut each of them,
towards zero, 13 binary places below the first place of the largest of the eight (measured: beside a product of 2^16 one
of 2^3 is kept whole, one of 1.875 * 2^3 becomes 2^3, one of 2^2 is lost; beside one of 1.875^2 * 2^14 one of 2^1 is kept;
in another group of eight any is).  The largest itself, of 8 significant places, is not cut.  So a group is off by less
than 7 * 2^-13 of its largest product, which is at most the product of the largest values of both sides there (`cut`)."""
import ctypes as C
import math

import pytest
import torch

from paper_2510_27656_amd import flmoe

U = 2.0 ** -23
BF16 = 2.0 ** -8
TINY = 2.0 ** -120           # below it bf16 and fp32 have subnormal steps; no value tested lies there
SLOPE = 1.2                  # no activation here is steeper (silu 1.0999, gelu 1.1289)


def config(counts, hidden=256, cap=0, max_tokens=None, top_k=1, align=1):
    n, el = len(counts), len(counts[0])
    tokens = max_tokens or max(1, max(sum(c) for c in counts))
    return flmoe.fl_moe_config(n, n * el, tokens, top_k, hidden, 0, align, 0, 0, cap, 0, 0, 0)


# ------------------------------------------------------------------ refusals (no GPU)
P = 0x10000                  # an aligned address that no refused call looks at


def calls():
    c = config([[4, 4], [4, 4]], hidden=256)
    at = [C.byref(c), 0, 2, P, P]
    return {
        "fl_moe_expert_gated": at + [128, 0] + [P, P, P, None, None, None],
        "fl_moe_expert_gated_backward": at + [128, 0] + [P, P, P, None, P, P + 16, P, P, None, None],
        "fl_moe_expert_product": at + [128, 256] + [P, P, P, None],
        "fl_moe_expert_product_backward": at + [128, 256] + [P, P, P, P, P, None],
        "fl_moe_expert_gated_e4m3": at + [128, 0] + [P, P, P, P, P, P, None],
        "fl_moe_expert_product_e4m3": at + [128, 256] + [P, P, P, P, P, None],
    }


INVALID, ALIGNMENT = flmoe.FL_ERR_INVALID_ARG, flmoe.FL_ERR_ALIGNMENT


def refused(name, code, **changed):
    args = calls()[name]
    for place, v in changed.items():
        args[int(place[1:])] = v
    assert getattr(flmoe.lib(), name)(*args) == code, changed


@pytest.mark.parametrize("name", sorted(calls()))
def test_ranges_tables_and_pointers_are_refused(name):
    refused(name, INVALID, a0=None)
    bad = config([[4, 4], [4, 4]])
    bad.top_k = 0
    refused(name, INVALID, a0=C.byref(bad))
    for begin, count in ((-1, 1), (0, 0), (0, 3), (2, 1), (1, 2), (0, -1), (1, 0x7fffffff)):
        refused(name, INVALID, a1=begin, a2=count)
    refused(name, INVALID, a3=None)
    refused(name, INVALID, a4=None)
    refused(name, ALIGNMENT, a3=P + 2)
    refused(name, ALIGNMENT, a4=P + 1)
    refused(name, INVALID, a5=0)
    refused(name, INVALID, a5=-8)
    refused(name, INVALID, a5=(1 << 20) + 128)
    refused(name, ALIGNMENT, a5=130)
    if "product" in name:
        refused(name, INVALID, a6=0)
        refused(name, INVALID, a6=(1 << 20) + 8)
        refused(name, ALIGNMENT, a6=257)
    else:
        refused(name, INVALID, a6=2)
        refused(name, INVALID, a6=-1)


@pytest.mark.parametrize("name,needed", [
    ("fl_moe_expert_gated", (7, 8, 9)), ("fl_moe_expert_gated_backward", (9, 11, 12)), ("fl_moe_expert_product", (7, 8, 9)),
    ("fl_moe_expert_product_backward", (9,)), ("fl_moe_expert_gated_e4m3", (7, 8, 9, 10, 11, 12)),
    ("fl_moe_expert_product_e4m3", (7, 8, 9, 10, 11))])
def test_missing_and_misaligned_tensors_are_refused(name, needed):
    for place in needed:
        refused(name, INVALID, **{f"a{place}": None})
        refused(name, ALIGNMENT, **{f"a{place}": P + 2})


def test_what_belongs_together_is_refused_apart():
    refused("fl_moe_expert_gated", INVALID, a11=P)                              # scales of nothing
    refused("fl_moe_expert_gated", ALIGNMENT, a10=P, a11=P, a5=136)             # blocks of 128 in a width of 136
    refused("fl_moe_expert_gated", ALIGNMENT, a10=P + 8)
    refused("fl_moe_expert_gated", ALIGNMENT, a10=P, a11=P + 1)
    back = "fl_moe_expert_gated_backward"
    refused(back, INVALID, a8=None)                                             # dx without w
    refused(back, INVALID, a7=None)                                             # dw without x
    refused(back, INVALID, a10=P, a12=P)                                        # 8-bit rows are no place for dpre
    refused(back, ALIGNMENT, a10=P, a5=136)
    for place in (7, 8, 13, 14, 15):
        refused(back, ALIGNMENT, **{f"a{place}": P + 8})
    back = "fl_moe_expert_product_backward"
    refused(back, INVALID, a10=None, a11=None)                                  # nothing wanted
    refused(back, INVALID, a8=None)
    refused(back, INVALID, a7=None)
    for place in (7, 8, 10, 11):
        refused(back, ALIGNMENT, **{f"a{place}": P + 8})
    refused("fl_moe_expert_gated_e4m3", ALIGNMENT, a0=C.byref(config([[4, 4], [4, 4]], hidden=264)))
    refused("fl_moe_expert_product_e4m3", ALIGNMENT, a5=136)


def test_the_binding_refuses_host_tensors():
    c = config([[4, 4]])
    z = torch.zeros(1 << 16, dtype=torch.bfloat16)
    t = torch.zeros(8, dtype=torch.int32)
    for call in (lambda: flmoe.fl_moe_expert_gated(c, 0, 1, t, t, 128, 0, z, z, z),
                 lambda: flmoe.fl_moe_expert_product(c, 0, 1, t, t, 128, 256, z, z, z),
                 lambda: flmoe.fl_moe_expert_product_backward(c, 0, 1, t, t, 128, 256, z, z, z, z)):
        with pytest.raises(flmoe.FlMoeError) as e:
            call()
        assert e.value.code == INVALID


# ------------------------------------------------------------------ on the GPU
class Layer:
    """Rows, tables and weights of one call.  Unused rows hold NaN: nothing may read a result out of them."""

    def __init__(self, counts, hidden, seed=0, cap=None, align=1, lead=0):
        self.counts, self.n, self.el, self.hidden = counts, len(counts), len(counts[0]), hidden
        off = []
        for per in counts:
            at, row = lead, [lead]
            for j, c in enumerate(per):
                at += -(-c // align) * align if j + 1 < len(per) else c
                row.append(at)
            off.append(row)
        self.off = off
        need = max(max(o) for o in off)
        self.cap = max(1, cap or need + 3)
        # as many tokens as the capacity needs: the configuration's own bound on rows
        self.cfg = config(counts, hidden, cap=self.cap, max_tokens=self.cap, align=1)
        assert flmoe.fl_moe_query_sizes(self.cfg).expert_capacity_rows == self.cap
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.expert_off = torch.tensor(off, dtype=torch.int32, device="cuda")
        self.loads = torch.tensor(counts, dtype=torch.int32, device="cuda")
        self.at = (self.cfg, 0, self.n, self.expert_off, self.loads)
        self.used = torch.zeros((self.n, self.cap), dtype=torch.bool, device="cuda")
        for d, j in self.experts():
            self.used[d, self.span(d, j)] = True

    def experts(self):
        return [(d, j) for d in range(self.n) for j in range(self.el)]

    def span(self, d, j):
        return slice(self.off[d][j], self.off[d][j] + self.counts[d][j])

    def randn(self, *shape, scale=1.0):
        return (torch.randn(shape, generator=self.g, device="cuda") * scale).to(torch.bfloat16)

    def rows(self, width, scale=1.0):
        r = self.randn(self.n, self.cap, width, scale=scale)
        r[~self.used] = math.nan
        return r

    def weights(self, out, in_):
        return self.randn(self.n * self.el, out, in_, scale=1 / math.sqrt(in_))

    def unwritten(self, width, dtype=torch.bfloat16):
        return torch.full((self.n, self.cap, width), 77, device="cuda").to(dtype)

    def check_rows(self, got, want, tolerance, what):
        """got within the tolerance of want(d, j) on every expert's rows, and as it was elsewhere."""
        for d, j in self.experts():
            if self.counts[d][j]:
                check(got[d, self.span(d, j)], want[d, j], tolerance[d, j], f"{what} of expert {d}, {j}")
        left = got[~self.used]
        assert bool((left == torch.full_like(left[:1], 77) if left.dtype != torch.float8_e4m3fn else left.float() == 77).all()), \
            f"{what}: a row of no expert was written"


def check(got, want, tolerance, what):
    got, off = got.double(), (got.double() - want).abs()
    bad = ~(off <= tolerance)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, the worst {float((off / tolerance).max()):.3g} times " \
        f"the tolerance, at {bad.nonzero()[0].tolist()}: {float(got[bad][0])} for {float(want[bad][0])}"


def act64(v, act):
    """activation, slope, and the argument of its exponential"""
    arg = v if act == 0 else 2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)
    s = torch.sigmoid(arg)
    inner = v if act == 0 else 2 * math.sqrt(2 / math.pi) * (v + 3 * 0.044715 * v ** 3)
    return v * s, s + inner * s * (1 - s), arg


def act_off(v, act, dv):
    """How far the activation of v, itself off by dv, may be: the exponential is good to a few units and to its argument's
    rounding."""
    a, _, arg = act64(v, act)
    return SLOPE * dv + (a.abs() + dv) * U * (16 + 8 * arg.abs())


def gated64(x, w, act, steps=None, off=0.0):
    """g, u, h and how far fp32 sums of `steps` additions (and `off` besides) leave g, u, h off, before rounding."""
    i = w.shape[0] // 2
    p, size = x @ w.T, x.abs() @ w.abs().T
    dp = (steps or x.shape[1]) * U * size + off
    g, u, dg, du = p[:, :i], p[:, i:], dp[:, :i], dp[:, i:]
    a = act64(g, act)[0]
    da = act_off(g, act, dg)
    return p, dp, a * u, da * (u.abs() + du) + a.abs() * du + 2 * U * (a * u).abs()


# no rows, one, fewer and more than any tile, a whole tile and its neighbours
SHAPES = [
    ([[1]], 8, 8), ([[3, 0]], 72, 40), ([[16, 17, 0, 1], [0, 0, 0, 0], [5, 0, 31, 33]], 256, 128),
    ([[64, 65]], 264, 136), ([[127, 128, 129]], 520, 264), ([[255, 0, 257], [256, 2, 511]], 200, 392),
    ([[700, 40]], 1032, 648), ([[9, 1000]], 2048, 96),
]


@pytest.mark.gpu
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("keep", ["nothing", "bf16", "e4m3"])
@pytest.mark.parametrize("counts,hidden,inter", SHAPES)
def test_gated(counts, hidden, inter, keep, act):
    if keep == "e4m3":
        inter = -(-inter // 128) * 128
    L = Layer(counts, hidden, align=16 if len(counts) > 1 else 1)
    x, w, h = L.rows(hidden), L.weights(2 * inter, hidden), L.unwritten(inter)
    pre = {"nothing": None, "bf16": L.unwritten(2 * inter), "e4m3": L.unwritten(2 * inter, torch.float8_e4m3fn)}[keep]
    scales = L.unwritten(2 * inter // 128, torch.float32) if keep == "e4m3" else None
    if keep == "e4m3":
        pre.view(torch.uint8).fill_(0)
        pre.copy_(torch.full_like(pre.float(), 77).to(pre.dtype))
    flmoe.fl_moe_expert_gated(*L.at, inter, act, x, w, h, pre, scales)
    want, tol, kept, kept_tol = {}, {}, {}, {}
    for d, j in L.experts():
        p, dp, h64, dh = gated64(x[d, L.span(d, j)].double(), w[d * L.el + j].double(), act)
        want[d, j], tol[d, j] = h64, h64.abs() * BF16 + (1 + BF16) * dh + TINY
        kept[d, j], kept_tol[d, j] = p, p.abs() * BF16 + (1 + BF16) * dp + TINY
    L.check_rows(h, want, tol, "h")
    if keep == "bf16":
        L.check_rows(pre, kept, kept_tol, "pre")
    if keep == "e4m3":
        check_blocks(L, pre, scales, kept, {e: t - kept[e].abs() * BF16 for e, t in kept_tol.items()}, "pre")


def check_blocks(L, codes, scales, want, off, what):
    """e4m3 blocks of want, itself off by `off` before it was quantised."""
    for d, j in L.experts():
        if not L.counts[d][j]:
            continue
        v, o = want[d, j].unflatten(1, (-1, 128)), off[d, j].unflatten(1, (-1, 128))
        s = scales[d, L.span(d, j)].double()[..., None]
        most, most_off = v.abs().amax(-1, keepdim=True), o.amax(-1, keepdim=True)
        check(s, most / 448, most / 448 * 2 * U + most_off / 448 + 2.0 ** -149, f"scales of {what} of expert {d}, {j}")
        got = codes[d, L.span(d, j)].float().double().unflatten(1, (-1, 128)) * s
        # half a step of the value (or of the smallest step), of the value as it was; the largest is held at 448 scales
        check(got, v, (v.abs() + o) * 2.0 ** -4 * (1 + 8 * U) + s * 2.0 ** -10 + o * (1 + 4 * U) + v.abs() * 4 * U + TINY, f"{what} of expert {d}, {j}")
    left = codes.float()[~L.used]
    assert bool((left == left[:1]).all()) and bool((scales[~L.used] == 77).all()), f"{what}: a row of no expert was written"


@pytest.mark.gpu
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("kept", ["bf16", "in place", "e4m3"])
@pytest.mark.parametrize("counts,hidden,inter", SHAPES)
def test_gated_backward(counts, hidden, inter, kept, act):
    """Every product against what it was given: dpre and h against pre, dx and dw against dpre."""
    if kept == "e4m3":
        inter = -(-inter // 128) * 128
    L = Layer(counts, hidden, align=16 if len(counts) > 1 else 1)
    x, w, dh = L.rows(hidden), L.weights(2 * inter, hidden), L.rows(inter)
    p = L.rows(2 * inter, scale=3.0)
    scales = None
    if kept == "e4m3":
        pre = (torch.randn(p.shape, generator=L.g, device="cuda") * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
        scales = torch.rand((L.n, L.cap, 2 * inter // 128), generator=L.g, device="cuda") / 50
        p64 = (pre.float().double().unflatten(2, (-1, 128)) * scales.double()[..., None]).flatten(2)
    else:
        pre, p64 = p, p.double()
    dpre = pre if kept == "in place" else L.unwritten(2 * inter)
    dx, h, dw = L.unwritten(hidden), L.unwritten(inter), torch.full_like(w, 77)
    flmoe.fl_moe_expert_gated_backward(*L.at, inter, act, x, w, pre, scales, dh, dpre, dx, dw, h)
    want, tol = {k: {} for k in ("dpre", "dx", "h")}, {k: {} for k in ("dpre", "dx", "h")}
    for d, j in L.experts():
        rows, e = L.span(d, j), d * L.el + j
        g, u = p64[d, rows, :inter], p64[d, rows, inter:]
        up = dh[d, rows].double()
        a, slope, arg = act64(g, act)
        da = act_off(g, act, g.abs() * U)
        # the slope: s and inner s (1 - s), s good to a few units and its argument's rounding
        dslope = (U * (16 + 8 * arg.abs())) * (1 + arg.abs() * 3)
        want["dpre"][d, j] = torch.cat((up * u * slope, up * a), 1)
        off = torch.cat(((up * u).abs() * (dslope + 4 * U), up.abs() * (da + 4 * U * a.abs())), 1)
        tol["dpre"][d, j] = want["dpre"][d, j].abs() * BF16 + (1 + BF16) * off + TINY
        want["h"][d, j] = a * u
        tol["h"][d, j] = (a * u).abs() * (BF16 + 4 * U) + (1 + BF16) * da * u.abs() + TINY
        dp, we = dpre[d, rows].double(), w[e].double()
        want["dx"][d, j] = dp @ we
        tol["dx"][d, j] = want["dx"][d, j].abs() * BF16 + (1 + BF16) * 2 * inter * U * (dp.abs() @ we.abs()) + TINY
        xe = x[d, rows].double()
        check(dw[e], dp.T @ xe, (dp.T @ xe).abs() * BF16 + (1 + BF16) * L.counts[d][j] * U * (dp.abs().T @ xe.abs()) + TINY, f"dw of expert {e}")
    if kept != "in place":
        L.check_rows(dpre, want["dpre"], tol["dpre"], "dpre")
    else:
        for d, j in L.experts():
            check(dpre[d, L.span(d, j)], want["dpre"][d, j], tol["dpre"][d, j], "dpre in place")
    L.check_rows(dx, want["dx"], tol["dx"], "dx")
    L.check_rows(h, want["h"], tol["h"], "h")


@pytest.mark.gpu
@pytest.mark.parametrize("counts,in_,out", SHAPES + [([[300]], 128, 8), ([[2, 2]], 4104, 16)])
def test_product_and_its_gradients(counts, in_, out):
    L = Layer(counts, 256)
    x, w, dy = L.rows(in_), L.weights(out, in_), L.rows(out)
    y, dx, dw = L.unwritten(out), L.unwritten(in_), torch.full_like(w, 77)
    flmoe.fl_moe_expert_product(*L.at, in_, out, x, w, y)
    flmoe.fl_moe_expert_product_backward(*L.at, in_, out, x, w, dy, dx, dw)
    want, tol = {"y": {}, "dx": {}}, {"y": {}, "dx": {}}
    for d, j in L.experts():
        rows, e = L.span(d, j), d * L.el + j
        xe, we, de = x[d, rows].double(), w[e].double(), dy[d, rows].double()
        want["y"][d, j], want["dx"][d, j] = xe @ we.T, de @ we
        tol["y"][d, j] = want["y"][d, j].abs() * BF16 + (1 + BF16) * in_ * U * (xe.abs() @ we.abs().T) + TINY
        tol["dx"][d, j] = want["dx"][d, j].abs() * BF16 + (1 + BF16) * out * U * (de.abs() @ we.abs()) + TINY
        check(dw[e], de.T @ xe, (de.T @ xe).abs() * BF16 + (1 + BF16) * L.counts[d][j] * U * (de.abs().T @ xe.abs()) + TINY, f"dw of expert {e}")
    L.check_rows(y, want["y"], tol["y"], "y")
    L.check_rows(dx, want["dx"], tol["dx"], "dx")
    # one gradient alone is the same gradient
    only = torch.full_like(w, 77)
    flmoe.fl_moe_expert_product_backward(*L.at, in_, out, x, None, dy, None, only)
    assert torch.equal(only, dw)
    only = L.unwritten(in_)
    flmoe.fl_moe_expert_product_backward(*L.at, in_, out, None, w, dy, only, None)
    assert torch.equal(only, dx)


def e4m3_rows(L, width):
    codes = (torch.randn((L.n, L.cap, width), generator=L.g, device="cuda") * 120).clamp(-448, 448).to(torch.float8_e4m3fn)
    scales = (torch.rand((L.n, L.cap, width // 128), generator=L.g, device="cuda") + 0.5) / 120
    codes.view(torch.uint8)[~L.used] = 0x7f                  # NaN
    scales[~L.used] = math.nan
    return codes, scales


def e4m3_weights(L, out, in_):
    e = L.n * L.el
    codes = (torch.randn((e, out, in_), generator=L.g, device="cuda") * 120).clamp(-448, 448).to(torch.float8_e4m3fn)
    scales = (torch.rand((e, -(-out // 128), in_ // 128), generator=L.g, device="cuda") + 0.5) / (120 * math.sqrt(in_))
    wide = scales.double().repeat_interleave(128, 1)[:, :out].repeat_interleave(128, 2)
    return codes, scales, codes.float().double() * wide


def dequantised(codes, scales):
    return codes.float().double() * scales.double().repeat_interleave(128, -1)


E4M3_SHAPES = [([[1]], 128, 128), ([[3, 0]], 256, 384), ([[16, 17, 0, 1], [0, 0, 0, 0], [5, 0, 31, 33]], 384, 128),
               ([[127, 128, 129]], 512, 256), ([[255, 0, 257], [256, 2, 511]], 256, 640), ([[9, 700]], 2048, 128)]


def cut(x, w):
    """What the matrix instruction may cut off the products' sums (see above)."""
    largest = lambda v: v.abs().unflatten(1, (-1, 8)).amax(-1)
    return 7 * 2.0 ** -13 * (largest(x) @ largest(w).T)


def sums(k):
    """Steps of a sum over e4m3 blocks: 128 products in a block, a multiplication of the scales, one addition a block."""
    return 128 + 3 + k // 128


@pytest.mark.gpu
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("counts,hidden,inter", E4M3_SHAPES)
def test_gated_e4m3(counts, hidden, inter, act):
    L = Layer(counts, hidden, align=16 if len(counts) > 1 else 1)
    (x, xs), (w, ws, w64) = e4m3_rows(L, hidden), e4m3_weights(L, 2 * inter, hidden)
    h, hs = L.unwritten(inter, torch.uint8).view(torch.float8_e4m3fn), L.unwritten(inter // 128, torch.float32)
    flmoe.fl_moe_expert_gated_e4m3(*L.at, inter, act, x, xs, w, ws, h, hs)
    want, off = {}, {}
    for d, j in L.experts():
        rows = L.span(d, j)
        x64, we = dequantised(x[d, rows], xs[d, rows]), w64[d * L.el + j]
        _, _, want[d, j], off[d, j] = gated64(x64, we, act, sums(hidden), cut(x64, we))
    check_blocks(L, h, hs, want, off, "h")


@pytest.mark.gpu
@pytest.mark.parametrize("counts,in_,out", E4M3_SHAPES + [([[300, 4]], 128, 8), ([[40]], 384, 392), ([[5]], 4096, 2056)])
def test_product_e4m3(counts, in_, out):
    L = Layer(counts, 256)
    (x, xs), (w, ws, w64) = e4m3_rows(L, in_), e4m3_weights(L, out, in_)
    y = L.unwritten(out)
    flmoe.fl_moe_expert_product_e4m3(*L.at, in_, out, x.view(torch.uint8), xs, w, ws, y)
    want, tol = {}, {}
    for d, j in L.experts():
        rows = L.span(d, j)
        x64, we = dequantised(x[d, rows], xs[d, rows]), w64[d * L.el + j]
        want[d, j] = x64 @ we.T
        tol[d, j] = want[d, j].abs() * BF16 + (1 + BF16) * (sums(in_) * U * (x64.abs() @ we.abs().T) + cut(x64, we)) + TINY
    L.check_rows(y, want, tol, "y")


@pytest.mark.gpu
def test_gradients_against_differences():
    """The sum of h dh along a direction, by the formula in 64 bits at two points, and by the kernels' gradients: off by
    what their entries may be off.  dpre is off by two roundings to bf16 (pre, dpre) and dx, dw by one more."""
    counts, hidden, inter = [[5, 33], [0, 70]], 136, 72
    for act in (0, 1):
        L = Layer(counts, hidden, seed=3)
        x, w, dh = L.rows(hidden), L.weights(2 * inter, hidden), L.rows(inter)
        h, pre, dpre, dx = L.unwritten(inter), L.unwritten(2 * inter), L.unwritten(2 * inter), L.unwritten(hidden)
        dw = torch.full_like(w, 77)
        flmoe.fl_moe_expert_gated(*L.at, inter, act, x, w, h, pre)
        flmoe.fl_moe_expert_gated_backward(*L.at, inter, act, x, w, pre, None, dh, dpre, dx, dw)
        for d, j in L.experts():
            rows, e = L.span(d, j), d * L.el + j
            xe, we, up = x[d, rows].double(), w[e].double(), dh[d, rows].double()

            def loss(a, b):
                p = a @ b.T
                return (act64(p[:, :inter], act)[0] * p[:, inter:] * up).sum()
            p, dp, _, _ = gated64(xe, we, act)
            g, u = p[:, :inter], p[:, inter:]
            a, slope, _ = act64(g, act)
            err = dp + p.abs() * BF16                       # of the kept pre-activations; no second derivative exceeds 1.6
            eg, eu = err[:, :inter], err[:, inter:]
            grad = torch.cat((up * u * slope, up * a), 1)
            off = torch.cat((up.abs() * (eu * SLOPE + (u.abs() + eu) * 1.6 * eg), up.abs() * SLOPE * eg), 1) + grad.abs() * BF16 * 1.1
            for got, point, error in ((dx[d, rows], 0, off @ we.abs()), (dw[e], 1, off.T @ xe.abs())):
                v = torch.randn(got.shape, generator=L.g, device="cuda", dtype=torch.float64)
                at = [xe, we]
                lo, hi = list(at), list(at)
                step = 1e-5
                lo[point], hi[point] = at[point] - step * v, at[point] + step * v
                difference = (loss(*hi) - loss(*lo)) / (2 * step)
                bound = (v.abs() * (error * 1.1 + got.double().abs() * BF16 * 1.1)).sum() + 1e-6
                assert abs(float((got.double() * v).sum() - difference)) <= float(bound), (act, e, point)


@pytest.mark.gpu
def test_calls_for_part_of_the_ranks_leave_the_others():
    counts, hidden, inter = [[40, 3], [7, 300], [0, 20], [1, 1]], 256, 128
    L = Layer(counts, hidden)
    x, w, dh = L.rows(hidden), L.weights(2 * inter, hidden), L.rows(inter)

    def run(ranges):
        h, pre, dpre, dx = L.unwritten(inter), L.unwritten(2 * inter), L.unwritten(2 * inter), L.unwritten(hidden)
        dw = torch.full_like(w, 77)
        for begin, count in ranges:
            at = (L.cfg, begin, count, L.expert_off, L.loads)
            flmoe.fl_moe_expert_gated(*at, inter, 0, x, w, h, pre)
            flmoe.fl_moe_expert_gated_backward(*at, inter, 0, x, w, pre, None, dh, dpre, dx, dw)
        return h, pre, dpre, dx, dw
    whole, parts, some = run([(0, 4)]), run([(2, 2), (0, 1), (1, 1)]), run([(1, 2)])
    for a, b, c in zip(whole, parts, some):
        assert torch.equal(a, b)
        per = c.shape[0] // 4
        assert torch.equal(c[per:3 * per], a[per:3 * per])
        for left in (c[:per], c[3 * per:]):
            assert bool((left == 77).all())


@pytest.mark.gpu
def test_rows_far_behind_the_start():
    """Rows whose offset passes 32 bits, in elements, in the last rows of a rank's capacity."""
    hidden, inter, cap = 32768, 128, 70000
    L = Layer([[5], [37]], hidden, cap=cap, lead=0)
    L.off = [[0, 5], [cap - 37, cap]]
    L.expert_off.copy_(torch.tensor(L.off))
    assert (2 * cap - 37) * hidden > 1 << 32
    x = torch.zeros((2, cap, hidden), dtype=torch.bfloat16, device="cuda")
    for d in (0, 1):
        x[d, L.span(d, 0)] = L.randn(L.counts[d][0], hidden)
    w = L.weights(2 * inter, hidden)
    dy, h, dx = torch.zeros((2, cap, inter), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, cap, inter), dtype=torch.bfloat16, device="cuda"), \
        torch.zeros_like(x)
    v, dv = L.weights(inter, hidden), torch.empty((2, inter, hidden), dtype=torch.bfloat16, device="cuda")
    flmoe.fl_moe_expert_gated(*L.at, inter, 0, x, w, h)
    for d in (0, 1):
        rows = L.span(d, 0)
        dy[d, rows] = L.randn(L.counts[d][0], inter)
        _, _, want, off = gated64(x[d, rows].double(), w[d].double(), 0)
        check(h[d, rows], want, want.abs() * BF16 + (1 + BF16) * off + TINY, "h")
    flmoe.fl_moe_expert_product_backward(*L.at, hidden, inter, x, v, dy, dx, dv)
    for d in (0, 1):
        rows = L.span(d, 0)
        de, ve, xe = dy[d, rows].double(), v[d].double(), x[d, rows].double()
        check(dx[d, rows], de @ ve, (de @ ve).abs() * BF16 + (1 + BF16) * inter * U * (de.abs() @ ve.abs()) + TINY, "dx")
        check(dv[d], de.T @ xe, (de.T @ xe).abs() * BF16 + (1 + BF16) * 37 * U * (de.abs().T @ xe.abs()) + TINY, "dw")


@pytest.mark.gpu
def test_tables_that_claim_too_much_stay_inside_the_capacity():
    """What a skipped step leaves in the tables: results are of no use, other memory is not touched."""
    hidden, inter = 256, 128
    L = Layer([[4, 4], [4, 4]], hidden, cap=16)
    x, w = torch.zeros((2, 16, hidden), dtype=torch.bfloat16, device="cuda"), L.weights(2 * inter, hidden)
    h = torch.full((2 * 16 + 8, inter), 77, dtype=torch.bfloat16, device="cuda")
    for off, loads in (([[0, 8, 16], [0, 8, 16]], [[4, 9], [100, 1 << 30]]), ([[-5, 16, 17], [1 << 30, -1, 3]], [[3, 3], [7, 7]]),
                       ([[0, 15, 16], [2, 3, 4]], [[-1, 5], [0x7fffffff, -0x80000000]])):
        flmoe.fl_moe_expert_gated(L.cfg, 0, 2, torch.tensor(off, dtype=torch.int32, device="cuda"),
                                  torch.tensor(loads, dtype=torch.int32, device="cuda"), inter, 0, x, w, h)
        torch.cuda.synchronize()
        assert bool((h[32:] == 77).all())


@pytest.mark.gpu
def test_infinities_and_nan_stay_in_their_rows():
    """A row that holds them answers with them; its neighbours, and in the weight gradient its neighbours' columns, do not."""
    counts, hidden, inter = [[20, 3]], 264, 136
    L = Layer(counts, hidden)
    x, w = L.rows(hidden), L.weights(2 * inter, hidden)
    h, clean = L.unwritten(inter), L.unwritten(inter)
    flmoe.fl_moe_expert_gated(*L.at, inter, 0, x, w, clean)
    x[0, 4, 263], x[0, 19, 0] = math.nan, math.inf
    flmoe.fl_moe_expert_gated(*L.at, inter, 0, x, w, h)
    fine = [r for r in range(23) if r not in (4, 19)]
    assert torch.equal(h[0, fine], clean[0, fine])
    assert bool(h[0, 4].isnan().all()) and not bool(h[0, 19].isfinite().any())
    dy, dw, before = L.rows(inter), torch.full((2, inter, hidden), 77, dtype=torch.bfloat16, device="cuda"), torch.empty((2, inter, hidden), dtype=torch.bfloat16, device="cuda")
    flmoe.fl_moe_expert_product_backward(*L.at, hidden, inter, L.rows(hidden), None, dy, None, before)
    flmoe.fl_moe_expert_product_backward(*L.at, hidden, inter, x, None, dy, None, dw)
    assert bool(dw[0, :, 263].isnan().all()) and not bool(dw[0, :, 0].isfinite().any())
    assert bool(dw[0, :, 1:263].isfinite().all()) and bool(dw[1].isfinite().all())


@pytest.mark.gpu
def test_blocks_with_infinities_and_nan():
    """e4m3 blocks of pre-activations: a NaN is skipped by the maximum, an Inf makes the scale infinite."""
    hidden = inter = 128
    L = Layer([[4]], hidden)
    x = torch.zeros((1, L.cap, hidden), dtype=torch.bfloat16, device="cuda")
    w = torch.zeros((1, 2 * inter, hidden), dtype=torch.bfloat16, device="cuda")
    w[0, :inter] = torch.eye(128, device="cuda")            # gates are the row itself
    x[0, 0, :3] = torch.tensor([448.0, -1.0, 0.5], device="cuda")
    x[0, 1, 0], x[0, 1, 1] = 896.0, -2.0
    h, pre, scales = L.unwritten(inter), L.unwritten(2 * inter, torch.uint8), L.unwritten(2, torch.float32)
    flmoe.fl_moe_expert_gated(*L.at, inter, 0, x, w, h, pre, scales)
    assert scales[0, :4, 0].tolist() == [1.0, 2.0, 1.0, 1.0] and scales[0, :4, 1].tolist() == [1.0] * 4
    assert pre[0, 0, :4].tolist() == [0x7e, 0xb8, 0x30, 0] and pre[0, 1, :3].tolist() == [0x7e, 0xb8, 0]
    # gates of inf and -inf among finite ones: 0 * inf elsewhere in the row is NaN
    x.zero_()
    x[0, 0, 5], x[0, 1, 5] = math.inf, -math.inf
    flmoe.fl_moe_expert_gated(*L.at, inter, 0, x, w, h, pre, scales)
    assert math.isinf(float(scales[0, 0, 0])) and math.isinf(float(scales[0, 1, 0]))
    assert int(pre[0, 0, 5]) == 0x7f and int(pre[0, 1, 5]) == 0xff
    assert bool(((pre[0, :2] & 0x7f) == 0x7f)[:, :128].all())


@pytest.mark.gpu
def test_runs_agree_bit_for_bit_also_on_another_stream_and_in_a_graph():
    counts, hidden, inter = [[40, 300], [513, 0]], 1024, 256
    L = Layer(counts, hidden)
    x, w, dh = L.rows(hidden), L.weights(2 * inter, hidden), L.rows(inter)
    (x8, xs), (w8, ws, _) = e4m3_rows(L, hidden), e4m3_weights(L, 2 * inter, hidden)
    v8, vs, _ = e4m3_weights(L, hidden, inter)

    def buffers():
        return [L.unwritten(inter), L.unwritten(2 * inter), L.unwritten(2 * inter), L.unwritten(hidden), torch.full_like(w, 77),
                L.unwritten(inter, torch.uint8), L.unwritten(inter // 128, torch.float32), L.unwritten(hidden)]

    def run(b, stream=None):
        h, pre, dpre, dx, dw, h8, hs, y = b
        flmoe.fl_moe_expert_gated(*L.at, inter, 0, x, w, h, pre, stream=stream)
        flmoe.fl_moe_expert_gated_backward(*L.at, inter, 0, x, w, pre, None, dh, dpre, dx, dw, stream=stream)
        flmoe.fl_moe_expert_gated_e4m3(*L.at, inter, 1, x8, xs, w8, ws, h8, hs, stream=stream)
        flmoe.fl_moe_expert_product_e4m3(*L.at, inter, hidden, h8, hs, v8, vs, y, stream=stream)
    first, second, third = buffers(), buffers(), buffers()
    run(first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    run(second, side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first, second):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        run(third)
    for seed in range(3):                            # new inputs in the same buffers, eager work between the replays
        x.copy_(L.rows(hidden))
        x8.view(torch.uint8)[L.used] = x8.view(torch.uint8)[L.used].flip(0)
        for t in third:
            t.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        run(first)
        for a, b in zip(first, third):
            assert torch.equal(a, b), seed


@pytest.mark.gpu
def test_the_binding_refuses_wrong_tensors():
    L = Layer([[4, 4]], 256)
    x, w, h = L.rows(256), L.weights(256, 256), L.unwritten(128)
    ok = (*L.at, 128, 0, x, w, h)
    flmoe.fl_moe_expert_gated(*ok)
    for place, bad in ((7, x.float()), (7, x[:, :-1]), (7, x.transpose(1, 2)), (8, w[:1]), (8, w.cpu()), (9, h[..., ::2]), (9, None),
                       (3, L.expert_off.long()), (4, L.loads[:, :1])):
        args = list(ok)
        args[place] = bad
        with pytest.raises(flmoe.FlMoeError) as e:
            flmoe.fl_moe_expert_gated(*args)
        assert e.value.code == INVALID, place


# ------------------------------------------------------------------ together with the shuffle
def layer_inputs(**kw):
    from paper_2510_27656_amd import harness, workloads
    wl = workloads.custom("layer", 4, 16, 37, 256, 4, seed=5, ragged=True, **kw)
    inp = workloads.make_inputs(wl)
    return wl, inp, harness.to_device(inp), harness


def tokens_by_expert(wl, inp):
    """(rank, token, slot) of the pairs of every expert, in the order of its rows: by source rank, then token."""
    pairs = {}
    for s in range(wl.n_ranks):
        for t in range(int(inp.num_tokens[s])):
            for k in range(wl.top_k):
                pairs.setdefault(int(inp.indices[s, t, k]), []).append((s, t, k))
    return pairs


@pytest.mark.gpu
@pytest.mark.parametrize("stream_ordered", [False, True])
def test_a_layer_of_bf16_tokens(stream_ordered):
    """dispatch, gated block, product, combine against the layer's formula in 64 bits, from the tokens to the sums."""
    wl, inp, dev, harness = layer_inputs()
    inter = 136
    sh = harness.make_shuffle(inp, stream_ordered=stream_ordered, expert_align=16)
    ex, (w, v) = harness.make_experts(sh, inter)
    out = harness.run_layer(sh, ex, (w, v), dev).clone()
    assert sh.status() == 0
    x = dev["x"].double()
    want, off = torch.zeros(out.shape, dtype=torch.float64, device="cuda"), torch.zeros(out.shape, dtype=torch.float64, device="cuda")
    for e, pairs in tokens_by_expert(wl, inp).items():
        s, t, k = (torch.tensor(c, device="cuda") for c in zip(*pairs))
        _, _, h, dh = gated64(x[s, t], w[e].double(), 0)
        dh = h.abs() * BF16 + (1 + BF16) * dh                # h is rounded to bf16
        y, size = h @ v[e].double().T, (h.abs() + dh) @ v[e].double().abs().T
        dy = dh @ v[e].double().abs().T + inter * U * size
        dy = y.abs() * BF16 + (1 + BF16) * dy                # and y
        g = dev["weights"][s, t, k].double()[:, None]
        want.index_put_((s, t), g * y, accumulate=True)
        off.index_put_((s, t), g.abs() * (dy + wl.top_k * U * (y.abs() + dy)), accumulate=True)
    for r in range(wl.n_ranks):
        n = int(inp.num_tokens[r])
        check(out[r, :n], want[r, :n], want[r, :n].abs() * BF16 + (1 + BF16) * off[r, :n] + TINY, f"out of rank {r}")
    sh.close()


@pytest.mark.gpu
def test_a_layer_of_e4m3_tokens():
    """The same with e4m3 dispatch: the rows are the oracle-checked codes, so the products are held against them."""
    wl, inp, dev, harness = layer_inputs(dispatch_dtype="e4m3")
    inter = 128
    sh = harness.make_shuffle(inp)
    ex, (w, v, ws, vs) = harness.make_experts(sh, inter)
    out = harness.run_layer(sh, ex, (w, v, ws, vs), dev)
    assert sh.status() == 0
    tabs = sh.layout_tables()
    wide = lambda c, s: c.float().double() * s.double().repeat_interleave(128, 1)[:, :c.shape[1]].repeat_interleave(128, 2)
    w64, v64 = wide(w, ws), wide(v, vs)
    x64 = dequantised(sh.expert_x.view(torch.float8_e4m3fn), sh.expert_scales)
    h64 = dequantised(ex.h.view(torch.float8_e4m3fn), ex.h_scales)
    for d in range(wl.n_ranks):
        for j in range(sh.El):
            lo, n, e = int(tabs["expert_off"][d, j]), int(tabs["G"][d, j]), d * sh.El + j
            rows = slice(lo, lo + n)
            _, _, h, dh = gated64(x64[d, rows], w64[e], 0, sums(wl.hidden), cut(x64[d, rows], w64[e]))
            s = ex.h_scales[d, rows].double().repeat_interleave(128, 1)
            check(h64[d, rows], h, (h.abs() + dh) * 2.0 ** -4 * (1 + 8 * U) + s * 2.0 ** -10 + dh + h.abs() * 4 * U + TINY, f"h of {e}")
            y = h64[d, rows] @ v64[e].T
            dy = sums(inter) * U * (h64[d, rows].abs() @ v64[e].abs().T) + cut(h64[d, rows], v64[e])
            check(ex.y[d, rows], y, y.abs() * BF16 + (1 + BF16) * dy + TINY, f"y of {e}")
    for r in range(wl.n_ranks):
        assert bool(out[r, :int(inp.num_tokens[r])].isfinite().all())
    sh.close()


@pytest.mark.gpu
@pytest.mark.parametrize("keep", ["bf16", "e4m3"])
def test_a_training_step_of_a_layer(keep):
    """Forward, another layer's step in between, backward: every gradient against the formula on what the layer kept, from
    the sums' gradient to the tokens'."""
    wl, inp, dev, harness = layer_inputs()
    inter = 128
    sh = harness.make_shuffle(inp)
    ex, (w, v) = harness.make_experts(sh, inter, training=True, keep=keep)
    harness.run_layer(sh, ex, (w, v), dev)
    x = sh.expert_x.clone()
    off, load = (t.cpu() for t in ex.tables)
    kept = ex.pre.clone()
    kept64 = dequantised(kept.view(torch.float8_e4m3fn), ex.pre_scales) if keep == "e4m3" else kept.double()
    other = dict(dev, indices=(dev["indices"] + 5) % wl.n_experts)
    pairs = tokens_by_expert(wl, inp)
    row_weights = torch.zeros((sh.N, sh.expert_capacity_rows), device="cuda")
    for e, p in pairs.items():
        d, j = e // sh.El, e % sh.El
        s, t, k = (torch.tensor(c, device="cuda") for c in zip(*p))
        row_weights[d, int(off[d, j]):int(off[d, j]) + len(p)] = dev["weights"][s, t, k]
        assert len(p) == int(load[d, j])
    harness.run_step(sh, other)              # another layer, with other routing, uses the same shuffle
    g = torch.Generator(device="cuda").manual_seed(1)
    dout = torch.randn(sh.out.shape, generator=g, device="cuda").to(torch.bfloat16)
    dw, dv = torch.full_like(w, 77), torch.full_like(v, 77)
    dx = harness.run_layer_backward(sh, ex, (w, v), (dw, dv), dev, x, dout, row_weights, torch.ones_like(dev["weights"]))
    assert sh.status() == 0
    dy64 = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    for e, p in pairs.items():
        d, j = e // sh.El, e % sh.El
        s, t, k = (torch.tensor(c, device="cuda") for c in zip(*p))
        dy64[d, int(off[d, j]):int(off[d, j]) + len(p)] = (dout[s, t].float() * dev["weights"][s, t, k][:, None]).to(torch.bfloat16).double()
    for e in range(wl.n_experts):
        d, j = e // sh.El, e % sh.El
        n = int(load[d, j])
        rows = slice(int(off[d, j]), int(off[d, j]) + n)
        xe, dy, p = x[d, rows].double(), dy64[d, rows], kept64[d, rows]
        a, slope, _ = act64(p[:, :inter], 0)
        h = ex.h[d, rows].double()
        bound = lambda want, size, steps: want.abs() * BF16 + (1 + BF16) * steps * U * size + TINY
        if keep == "e4m3":
            check(h, a * p[:, inter:], (a * p[:, inter:]).abs() * (BF16 + 64 * U) + TINY, f"h again of {e}")
        check(dv[e], dy.T @ h, bound(dy.T @ h, dy.abs().T @ h.abs(), n), f"dw_out of {e}")
        dh = ex.dh[d, rows].double()
        check(dh, dy @ v[e].double(), bound(dy @ v[e].double(), dy.abs() @ v[e].double().abs(), wl.hidden), f"dh of {e}")
        dp = ex.dpre[d, rows].double()
        want = torch.cat((dh * p[:, inter:] * slope, dh * a), 1)
        check(dp, want, want.abs() * BF16 + (dh.abs() * (1 + p[:, inter:].abs())).repeat(1, 2) * U * 128 + TINY, f"dpre of {e}")
        check(dw[e], dp.T @ xe, bound(dp.T @ xe, dp.abs().T @ xe.abs(), n), f"dw_in of {e}")
        check(ex.dx[d, rows], dp @ w[e].double(), bound(dp @ w[e].double(), dp.abs() @ w[e].double().abs(), 2 * inter), f"dx of {e}")
    # the tokens' gradient: sums over a token's rows of dx, in fp32 in the order of k, rounded once
    sums_of = torch.zeros(dx.shape, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(sums_of)
    for e, p in pairs.items():
        d, j = e // sh.El, e % sh.El
        s, t, k = (torch.tensor(c, device="cuda") for c in zip(*p))
        r = ex.dx[d, int(off[d, j]):int(off[d, j]) + len(p)].double()
        sums_of.index_put_((s, t), r, accumulate=True)
        size.index_put_((s, t), r.abs(), accumulate=True)
    for r in range(wl.n_ranks):
        n = int(inp.num_tokens[r])
        check(dx[r, :n], sums_of[r, :n], sums_of[r, :n].abs() * BF16 + (1 + BF16) * wl.top_k * U * size[r, :n] + TINY, f"dx of rank {r}")
    sh.close()


@pytest.mark.gpu
def test_rows_of_e4m3_have_no_backward_pass():
    wl, inp, dev, harness = layer_inputs(dispatch_dtype="e4m3")
    sh = harness.make_shuffle(inp)
    with pytest.raises(flmoe.FlMoeError):
        flmoe.MoEExperts(sh, 128, training=True)
    with pytest.raises(flmoe.FlMoeError):
        flmoe.MoEExperts(sh, 128, keep="fp8")
    sh.close()


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [[[300, 70, 5]], [[64, 65], [33, 31]], [[1, 900]]])
@pytest.mark.parametrize("tokens", [1, 30, 100000])
def test_tiles_chosen_for_other_numbers_of_rows_are_right_too(tokens, counts):
    """The tile goes by the mean that the configuration expects: few rows where many were meant, and the other way round."""
    hidden, inter = 384, 256
    L = Layer(counts, hidden)
    cap = L.cap
    L.cfg.max_tokens, L.cfg.top_k = max(tokens * L.el, 1), 1
    sizes = flmoe.fl_moe_query_sizes(L.cfg)
    if sizes.expert_capacity_rows != cap:                    # the configuration holds fewer rows than these tensors
        L = Layer([[min(c, tokens) for c in per] for per in counts], hidden, cap=sizes.expert_capacity_rows)
        L.cfg.max_tokens, L.cfg.top_k = max(tokens * L.el, 1), 1
    at = (L.cfg, 0, L.n, L.expert_off, L.loads)
    x, w, h = L.rows(hidden), L.weights(2 * inter, hidden), L.unwritten(inter)
    v, y = L.weights(hidden, inter), L.unwritten(hidden)
    (x8, xs), (w8, ws, w64) = e4m3_rows(L, hidden), e4m3_weights(L, 2 * inter, hidden)
    h8, hs = L.unwritten(inter, torch.uint8).view(torch.float8_e4m3fn), L.unwritten(inter // 128, torch.float32)
    pre, ps = L.unwritten(2 * inter, torch.uint8).view(torch.float8_e4m3fn), L.unwritten(2 * inter // 128, torch.float32)
    h2 = L.unwritten(inter)
    flmoe.fl_moe_expert_gated(*at, inter, 0, x, w, h)
    flmoe.fl_moe_expert_gated(*at, inter, 0, x, w, h2, pre, ps)
    assert torch.equal(h, h2)
    flmoe.fl_moe_expert_product(*at, inter, hidden, h, v, y)
    flmoe.fl_moe_expert_gated_e4m3(*at, inter, 0, x8, xs, w8, ws, h8, hs)
    want, tol, ywant, ytol, want8, off8, kept, kept_off = ({} for _ in range(8))
    for d, j in L.experts():
        rows, e = L.span(d, j), d * L.el + j
        p, dp, h64, dh = gated64(x[d, rows].double(), w[e].double(), 0)
        want[d, j], tol[d, j] = h64, h64.abs() * BF16 + (1 + BF16) * dh + TINY
        kept[d, j], kept_off[d, j] = p, dp
        he = h[d, rows].double()
        ywant[d, j] = he @ v[e].double().T
        ytol[d, j] = ywant[d, j].abs() * BF16 + (1 + BF16) * inter * U * (he.abs() @ v[e].double().abs().T) + TINY
        x64 = dequantised(x8[d, rows], xs[d, rows])
        _, _, want8[d, j], off8[d, j] = gated64(x64, w64[e], 0, sums(hidden), cut(x64, w64[e]))
    L.check_rows(h, want, tol, "h")
    L.check_rows(y, ywant, ytol, "y")
    check_blocks(L, h8, hs, want8, off8, "h in e4m3")
    check_blocks(L, pre, ps, kept, kept_off, "pre in e4m3")


# experts of some whole tiles of rows and a rest, among many of few rows or none; one of nearly all rows
UNEVEN = [
    [[(1024 + rest if j % 5 == 0 else j % 4) for j in range(70) for rest in ((1, 64, 128, 129, 255, 256, 0)[j // 5 % 7],)]],
    [[0] * 40 + [1152] + [1] * 4, [0] * 44 + [1281], [2] * 44 + [1300]],
    [[5000] + [0] * 62 + [1, 7]],
]


@pytest.mark.gpu
@pytest.mark.parametrize("counts", UNEVEN)
def test_tiles_of_uneven_experts_are_each_done_once(counts):
    """More tiles than workgroups and shares that differ: the last tiles of long experts come behind all others, and the weight
    gradients' shares go by the experts' rows."""
    in_, out = 512, 776
    L = Layer(counts, in_)
    x, w, dy = L.rows(in_), L.weights(out, in_), L.rows(out)
    y, dx, dw = L.unwritten(out), L.unwritten(in_), torch.full_like(w, 77)
    (x8, xs), (w8, ws, w64) = e4m3_rows(L, in_), e4m3_weights(L, out, in_)
    y8 = L.unwritten(out)
    flmoe.fl_moe_expert_product(*L.at, in_, out, x, w, y)
    flmoe.fl_moe_expert_product_backward(*L.at, in_, out, x, w, dy, dx, dw)
    flmoe.fl_moe_expert_product_e4m3(*L.at, in_, out, x8.view(torch.uint8), xs, w8, ws, y8)
    want, tol = {"y": {}, "dx": {}, "y8": {}}, {"y": {}, "dx": {}, "y8": {}}
    for d, j in L.experts():
        rows, e = L.span(d, j), d * L.el + j
        xe, we, de = x[d, rows].double(), w[e].double(), dy[d, rows].double()
        want["y"][d, j], want["dx"][d, j] = xe @ we.T, de @ we
        tol["y"][d, j] = want["y"][d, j].abs() * BF16 + (1 + BF16) * in_ * U * (xe.abs() @ we.abs().T) + TINY
        tol["dx"][d, j] = want["dx"][d, j].abs() * BF16 + (1 + BF16) * out * U * (de.abs() @ we.abs()) + TINY
        check(dw[e], de.T @ xe, (de.T @ xe).abs() * BF16 + (1 + BF16) * L.counts[d][j] * U * (de.abs().T @ xe.abs()) + TINY, f"dw of expert {e}")
        x64, we = dequantised(x8[d, rows], xs[d, rows]), w64[e]
        want["y8"][d, j] = x64 @ we.T
        tol["y8"][d, j] = want["y8"][d, j].abs() * BF16 + (1 + BF16) * (sums(in_) * U * (x64.abs() @ we.abs().T) + cut(x64, we)) + TINY
    for name, got in (("y", y), ("dx", dx), ("y8", y8)):
        L.check_rows(got, want[name], tol[name], name)


@pytest.mark.gpu
def test_a_layer_rank_by_rank_keeps_each_ranks_own_tables():
    """As a real rank calls it, streams given as handles: the others' tables, which may be in the making, are left alone."""
    wl, inp, dev, harness = layer_inputs()
    sh = harness.make_shuffle(inp)
    ex, (w, v) = harness.make_experts(sh, 128, training=True)
    harness.run_layer(sh, ex, (w, v), dev)
    y, tables = ex.y.clone(), [t.clone() for t in ex.tables]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for r in range(wl.n_ranks):
        ex.y.fill_(77)
        for t in ex.tables:
            t.fill_(-5)
        stream.wait_stream(torch.cuda.current_stream())
        ex.forward(w, v, ranks=(r, 1), stream=stream.cuda_stream)
        stream.synchronize()
        for d in range(wl.n_ranks):
            for mine, whole in zip(ex.tables, tables):
                assert torch.equal(mine[d], whole[d] if d == r else torch.full_like(whole[d], -5))
            for j in range(sh.El):
                rows = slice(int(tables[0][d, j]), int(tables[0][d, j] + tables[1][d, j]))
                assert torch.equal(ex.y[d, rows], y[d, rows] if d == r else torch.full_like(y[d, rows], 77))
    sh.close()


@pytest.mark.gpu
def test_other_rows_of_e4m3_come_with_their_scales():
    wl, inp, dev, harness = layer_inputs(dispatch_dtype="e4m3")
    sh = harness.make_shuffle(inp)
    ex, weights = harness.make_experts(sh, 128)
    harness.run_layer(sh, ex, weights, dev)
    y, x, scales = ex.y.clone(), sh.expert_x.clone(), sh.expert_scales.clone()
    harness.run_step(sh, dev)
    sh.expert_x.fill_(0x7f)
    for given in (dict(x=x), dict(x_scales=scales)):
        with pytest.raises(flmoe.FlMoeError):
            ex.forward(*weights, **given)
    off, load = (sh.layout_tables()[t].cpu() for t in ("expert_off", "G"))
    again = ex.forward(*weights, x=x, x_scales=scales)
    for d in range(wl.n_ranks):
        for j in range(sh.El):
            rows = slice(int(off[d, j]), int(off[d, j] + load[d, j]))
            assert torch.equal(again[d, rows], y[d, rows])
    sh.close()


@pytest.mark.gpu
def test_no_backward_pass_of_what_was_not_kept():
    wl, inp, dev, harness = layer_inputs()
    sh = harness.make_shuffle(inp)
    ex, (w, v) = harness.make_experts(sh, 128)
    harness.run_layer(sh, ex, (w, v), dev)
    with pytest.raises(flmoe.FlMoeError):
        ex.backward(ex.y, w, v, torch.empty_like(w), torch.empty_like(v))
    sh.close()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,hidden", [(16, 2056), (40, 2056), (16, 1024), (128, 1096)])
def test_a_sums_order_goes_by_the_expert_and_its_rows_alone(rows, hidden):
    """Tiles of few rows begin their sums at different steps of the contraction.  Where goes by the expert and the features: not
    by what is kept for the backward pass, by the ranks that a call is for, or by the other experts' rows."""
    n, el, inter = 8, 16, 256
    counts = [[max(0, rows - (7 * j + 3 * d) % 5) for j in range(el)] for d in range(n)]
    counts[2][3], counts[5][0] = 0, 1
    L = Layer(counts, hidden)
    assert abs(L.cfg.max_tokens // el - rows) <= 4           # the mean that the tile is chosen by
    x, w, v = L.rows(hidden), L.weights(2 * inter, hidden), L.weights(hidden, inter)
    wide = -(-hidden // 128) * 128
    (x8, xs), (w8, ws, w64) = e4m3_rows(L, wide), e4m3_weights(L, inter, wide)

    def run(ranges, keep, loads):
        h, y, y8 = L.unwritten(inter), L.unwritten(hidden), L.unwritten(inter)
        pre = {"nothing": None, "bf16": L.unwritten(2 * inter), "e4m3": L.unwritten(2 * inter, torch.uint8)}[keep]
        scales = L.unwritten(2 * inter // 128, torch.float32) if keep == "e4m3" else None
        for begin, count in ranges:
            at = (L.cfg, begin, count, L.expert_off, loads)
            flmoe.fl_moe_expert_gated(*at, inter, 0, x, w, h, pre, scales)
            flmoe.fl_moe_expert_product(*at, inter, hidden, h, v, y)
            flmoe.fl_moe_expert_product_e4m3(*at, wide, inter, x8, xs, w8, ws, y8)
        return h, y, y8
    whole = run([(0, n)], "nothing", L.loads)
    want, tol = ({k: {} for k in ("h", "y", "y8")} for _ in range(2))
    for d, j in L.experts():
        at, e = L.span(d, j), d * el + j
        _, _, h64, dh = gated64(x[d, at].double(), w[e].double(), 0)
        want["h"][d, j], tol["h"][d, j] = h64, h64.abs() * BF16 + (1 + BF16) * dh + TINY
        he, ve = whole[0][d, at].double(), v[e].double()
        want["y"][d, j] = he @ ve.T
        tol["y"][d, j] = want["y"][d, j].abs() * BF16 + (1 + BF16) * inter * U * (he.abs() @ ve.abs().T) + TINY
        x64 = dequantised(x8[d, at], xs[d, at])
        want["y8"][d, j] = x64 @ w64[e].T
        tol["y8"][d, j] = want["y8"][d, j].abs() * BF16 + (1 + BF16) * (sums(wide) * U * (x64.abs() @ w64[e].abs().T) + cut(x64, w64[e])) + TINY
    for name, got in zip(("h", "y", "y8"), whole):
        L.check_rows(got, want[name], tol[name], name)
    for keep in ("nothing", "bf16", "e4m3"):
        for got, first in zip(run([(0, n)], keep, L.loads), whole):
            assert torch.equal(got, first), keep
        for got, first in zip(run([(r, 1) for r in range(n)], keep, L.loads), whole):
            assert torch.equal(got, first), (keep, "rank by rank")
    fewer = L.loads.clone()                                  # the other experts' rows: half of the experts have none
    fewer.view(-1)[::2] = 0
    for got, first in zip(run([(0, n)], "nothing", fewer), whole):
        for d, j in L.experts():
            if int(fewer[d, j]):
                assert torch.equal(got[d, L.span(d, j)], first[d, L.span(d, j)]), (d, j)


@pytest.mark.gpu
def test_blocks_of_values_too_small_for_a_scale_are_zeros():
    """The largest product of a block is 2^-145: over 448 it is 0, no scale that its zeros could be divided by."""
    hidden = inter = 128
    L = Layer([[3]], hidden)
    x = torch.zeros((1, L.cap, hidden), device="cuda")
    w = torch.zeros((1, 2 * inter, hidden), device="cuda")
    x[0, 0, 0] = w[0, 5, 0] = w[0, inter + 5, 0] = 1.0
    x, w = x.to(torch.float8_e4m3fn), w.to(torch.float8_e4m3fn)
    xs = torch.ones((1, L.cap, 1), device="cuda")
    ws = torch.tensor([2.0 ** -70, 2.0 ** -74], device="cuda").view(1, 2, 1)     # silu(2^-70) = 2^-71
    h, hs, y = L.unwritten(inter, torch.uint8), L.unwritten(1, torch.float32), L.unwritten(hidden)
    flmoe.fl_moe_expert_gated_e4m3(*L.at, inter, 0, x, xs, w, ws, h, hs)
    assert hs[0, :3, 0].tolist() == [1.0, 1.0, 1.0]
    assert not bool((h[0, :3] & 0x7f).any())
    v = torch.ones((1, hidden, inter), device="cuda").to(torch.float8_e4m3fn)
    flmoe.fl_moe_expert_product_e4m3(*L.at, inter, hidden, h, hs, v, torch.ones((1, 1, 1), device="cuda"), y)
    assert not bool(y[0, :3].any())


@pytest.mark.gpu
@pytest.mark.parametrize("keep", ["bf16", "e4m3"])
def test_a_backward_pass_needs_what_a_forward_pass_kept(keep):
    """With bf16 it takes the place of what was kept: a second one, of all ranks or of one that has had its own, is refused.  What
    was kept in 8 bits stays."""
    wl, inp, dev, harness = layer_inputs()
    sh = harness.make_shuffle(inp)
    ex, (w, v) = harness.make_experts(sh, 128, training=True, keep=keep)
    dy = torch.randn(ex.y.shape, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(torch.bfloat16)

    def backward(ranks=None):
        dw, dv = torch.zeros_like(w), torch.zeros_like(v)
        dx = ex.backward(dy, w, v, dw, dv, ranks=ranks)
        return dw, dv, dx.clone()

    def refused(ranks=None):
        with pytest.raises(flmoe.FlMoeError) as e:
            backward(ranks)
        assert e.value.code == INVALID

    def used(dx):
        off, load = (t.cpu() for t in ex.tables)
        return torch.cat([dx[d, int(off[d, j]):int(off[d, j] + load[d, j])] for d in range(sh.N) for j in range(sh.El)])
    refused()                                                # no forward pass yet
    harness.run_layer(sh, ex, (w, v), dev)
    with pytest.raises(flmoe.FlMoeError):                    # a call that is refused for its tensors takes nothing away
        ex.backward(dy, w, v, torch.zeros_like(w)[:1], torch.zeros_like(v))
    dw, dv, dx = backward()
    if keep == "e4m3":
        for a, b in zip(backward()[:2], (dw, dv)):
            assert torch.equal(a, b)
        sh.close()
        return
    refused()
    ex.forward(w, v, ranks=(1, 2))
    refused()
    refused((0, 2))
    parts = backward((2, 1))
    refused((2, 1))
    refused((1, 2))
    for a, b in zip(parts[:2], (dw, dv)):
        assert torch.equal(a[2 * sh.El:3 * sh.El], b[2 * sh.El:3 * sh.El])
    backward((1, 1))
    # the forward pass from a graph: its replays are not seen, so nothing is refused
    ex.forward(w, v)
    backward()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ex.forward(w, v)
    for _ in range(3):
        graph.replay()
        again = backward()
        torch.cuda.synchronize()
        assert torch.equal(again[0], dw) and torch.equal(again[1], dv) and torch.equal(used(again[2]), used(dx))
    sh.close()


@pytest.mark.gpu
def test_both_passes_of_the_experts_in_one_graph():
    wl, inp, dev, harness = layer_inputs()
    sh = harness.make_shuffle(inp)
    ex, (w, v) = harness.make_experts(sh, 128, training=True)
    harness.run_layer(sh, ex, (w, v), dev)
    dy, dw, dv = ex.y.clone(), torch.zeros_like(w), torch.zeros_like(v)
    ex.backward(dy, w, v, dw, dv)
    want = dw.clone(), dv.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ex.forward(w, v)
        ex.backward(dy, w, v, dw, dv)
    for _ in range(3):
        dw.fill_(77)
        dv.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dw, want[0]) and torch.equal(dv, want[1])
    sh.close()


@pytest.mark.gpu
def test_other_activations_are_refused():
    wl, inp, dev, harness = layer_inputs()
    sh = harness.make_shuffle(inp)
    with pytest.raises(flmoe.FlMoeError) as e:
        flmoe.MoEExperts(sh, 128, activation="relu")
    assert e.value.code == INVALID
    sh.close()


def expert_rows(sh, wl, inp, dev, off, load):
    """The routing weights of the expert rows, and [(s, t, rank, rows)] of every expert's pairs."""
    weights, places = torch.zeros((sh.N, sh.expert_capacity_rows), device="cuda"), []
    for e, p in tokens_by_expert(wl, inp).items():
        d, j = e // sh.El, e % sh.El
        assert len(p) == int(load[d, j])
        s, t, k = (torch.tensor(c, device="cuda") for c in zip(*p))
        rows = slice(int(off[d, j]), int(off[d, j]) + len(p))
        weights[d, rows] = dev["weights"][s, t, k]
        places.append((s, t, d, rows))
    return weights, places


@pytest.mark.gpu
def test_a_training_step_of_a_layer_with_partial_sums():
    """The tokens' gradients come back as one row of each rank: the rank's sum of fp32, rounded, then the sum of those."""
    wl, inp, dev, harness = layer_inputs()
    sh = harness.make_shuffle(inp, partial_sums=True)
    ex, (w, v) = harness.make_experts(sh, 128, training=True)
    harness.run_layer(sh, ex, (w, v), dev)
    x, (off, load) = sh.expert_x.clone(), (t.cpu() for t in ex.tables)
    row_weights, places = expert_rows(sh, wl, inp, dev, off, load)
    dout = torch.randn(sh.out.shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    dw, dv = torch.full_like(w, 77), torch.full_like(v, 77)
    dx = harness.run_layer_backward(sh, ex, (w, v), (dw, dv), dev, x, dout, row_weights, torch.ones_like(dev["weights"]))
    assert sh.status() == 0
    for (s, t, d, rows), e in zip(places, tokens_by_expert(wl, inp)):
        dy = (dout[s, t].float() * row_weights[d, rows, None]).to(torch.bfloat16).double()
        h, n = ex.h[d, rows].double(), len(s)
        check(dv[e], dy.T @ h, (dy.T @ h).abs() * BF16 + (1 + BF16) * n * U * (dy.abs().T @ h.abs()) + TINY, f"dw_out of {e}")
        dp, xe = ex.dpre[d, rows].double(), x[d, rows].double()
        check(dw[e], dp.T @ xe, (dp.T @ xe).abs() * BF16 + (1 + BF16) * n * U * (dp.abs().T @ xe.abs()) + TINY, f"dw_in of {e}")
    of_rank = torch.zeros((sh.N, *dx.shape), dtype=torch.float64, device="cuda")
    size = torch.zeros(dx.shape, dtype=torch.float64, device="cuda")
    for s, t, d, rows in places:
        of_rank[d].index_put_((s, t), ex.dx[d, rows].double(), accumulate=True)
        size.index_put_((s, t), ex.dx[d, rows].double().abs(), accumulate=True)
    off = of_rank.abs().sum(0) * BF16 + 2 * wl.top_k * U * size              # the ranks' sums are rounded
    for r in range(wl.n_ranks):
        n, want = int(inp.num_tokens[r]), of_rank.sum(0)[r]
        check(dx[r, :n], want[:n], want[:n].abs() * BF16 + (1 + BF16) * off[r, :n] + TINY, f"dx of rank {r}")
    sh.close()


@pytest.mark.gpu
def test_tokens_that_a_rank_does_not_have_get_no_gradient():
    wl, inp, dev, harness = layer_inputs()
    sh = harness.make_shuffle(inp)
    ex, (w, v) = harness.make_experts(sh, 128, training=True)
    harness.run_layer(sh, ex, (w, v), dev)
    row_weights, _ = expert_rows(sh, wl, inp, dev, *(t.cpu() for t in ex.tables))
    x, dout, ones = sh.expert_x.clone(), torch.zeros_like(sh.out), torch.ones_like(dev["weights"])
    before = [torch.full_like(sh.out, 77) for _ in range(4)]                 # what the allocator hands out next
    del before
    dx = harness.run_layer_backward(sh, ex, (w, v), (torch.empty_like(w), torch.empty_like(v)), dev, x, dout, row_weights, ones)
    assert min(inp.num_tokens) < wl.tokens and not bool(dx.any())
    sh.close()


@pytest.mark.gpu
@pytest.mark.parametrize("n,el,mean", [(4, 256, 4), (4, 256, 40), (40, 25, 100), (3, 171, 30)])
def test_more_experts_than_a_workgroup_has_threads(n, el, mean):
    """The counts are scanned in turns of 256 or 512; the last experts, alone and with all others, have their own rows."""
    in_, out = 128, 136
    counts = [[(j * 7 + d * 3) % (2 * mean + 1) for j in range(el)] for d in range(n)]
    counts[-1][-1] = mean + 300                              # more than one tile behind all others
    L = Layer(counts, in_)
    assert abs(L.cfg.max_tokens // el - mean) <= 15          # the mean that the tile is chosen by
    x, w, dy = L.rows(in_), L.weights(out, in_), L.rows(out)
    y, dx, dw, part = L.unwritten(out), L.unwritten(in_), torch.full_like(w, 77), L.unwritten(out)
    flmoe.fl_moe_expert_product(*L.at, in_, out, x, w, y)
    flmoe.fl_moe_expert_product_backward(*L.at, in_, out, x, w, dy, dx, dw)
    flmoe.fl_moe_expert_product(L.cfg, n - 1, 1, L.expert_off, L.loads, in_, out, x, w, part)
    assert torch.equal(part[n - 1], y[n - 1]) and bool((part[:n - 1] == 77).all())
    for d in range(n):                                       # a rank's experts in one batch, padded
        most = max(max(counts[d]), 1)
        at = torch.tensor([[L.off[d][j] + min(r, max(counts[d][j] - 1, 0)) for r in range(most)] for j in range(el)], device="cuda")
        there = (torch.arange(most, device="cuda")[None] < L.loads[d][:, None])[..., None]
        take = lambda rows: rows[d][at].double().masked_fill(~there, 0)
        xe, de, we = take(x), take(dy), w[d * el:(d + 1) * el].double()
        for got, a, b, steps in ((take(y), xe, we.transpose(1, 2).contiguous(), in_), (take(dx), de, we, out),
                                 (dw[d * el:(d + 1) * el].double(), de.transpose(1, 2).contiguous(), xe, most)):
            want, size = torch.bmm(a, b), torch.bmm(a.abs(), b.abs())
            check(got, want, want.abs() * BF16 + (1 + BF16) * steps * U * size + TINY, f"rank {d}")
    for got in (y, dx):
        assert bool((got[~L.used] == 77).all())


@pytest.mark.gpu
def test_codes_and_scales_that_are_not_finite_stay_in_their_rows():
    """NaN codes and infinite or NaN scales of rows that are in use: the row is NaN where they enter, its neighbours are not."""
    counts, in_, out = [[20, 3, 140]], 384, 264
    L = Layer(counts, in_)
    (x, xs), (w, ws, _) = e4m3_rows(L, in_), e4m3_weights(L, out, in_)
    y, clean = L.unwritten(out), L.unwritten(out)
    flmoe.fl_moe_expert_product_e4m3(*L.at, in_, out, x, xs, w, ws, clean)
    x.view(torch.uint8)[0, 4, 300], x.view(torch.uint8)[0, 160, 0] = 0x7f, 0xff
    xs[0, 19, 2], xs[0, 21, 0] = math.nan, math.inf
    flmoe.fl_moe_expert_product_e4m3(*L.at, in_, out, x, xs, w, ws, y)
    bad = [4, 160, 19, 21]
    fine = [r for r in range(163) if r not in bad]
    assert torch.equal(y[0, fine], clean[0, fine])
    assert bool(y[0, [4, 160, 19]].isnan().all()) and not bool(y[0, 21].isfinite().any())
    # in the weights: the features whose codes or block they are in, of that expert
    w.view(torch.uint8)[1, 200, 17] = 0x7f
    ws[2, 2, 1] = math.inf                                   # features 256 to 263
    x, xs = e4m3_rows(L, in_)
    flmoe.fl_moe_expert_product_e4m3(*L.at, in_, out, x, xs, w, ws, y)
    assert bool(y[0, :20].isfinite().all())
    one = torch.arange(out, device="cuda") == 200
    assert bool(y[0, 20:23, one].isnan().all()) and bool(y[0, 20:23, ~one].isfinite().all())
    assert bool(y[0, 23:163, :256].isfinite().all()) and not bool(y[0, 23:163, 256:].isfinite().any())
    # the gated block answers with blocks of NaN codes there, finite ones elsewhere
    hidden, inter = 384, 256
    (x, xs), (w, ws, _) = e4m3_rows(L, hidden), e4m3_weights(L, 2 * inter, hidden)
    x.view(torch.uint8)[0, 7, 100] = 0x7f
    h, hs = L.unwritten(inter, torch.uint8), L.unwritten(inter // 128, torch.float32)
    flmoe.fl_moe_expert_gated_e4m3(*L.at, inter, 0, x, xs, w, ws, h, hs)
    assert bool(((h[0, 7] & 0x7f) == 0x7f).all()) and bool((hs[0, 7] == 1).all())
    rest = [r for r in range(163) if r != 7]
    assert not bool(((h[0, rest] & 0x7f) == 0x7f).any()) and bool(hs[0, rest].isfinite().all())


@pytest.mark.gpu
def test_each_gradient_of_the_gated_block_alone():
    """dx, dw, both or neither: the same bits; dpre is there each time."""
    counts, hidden, inter = [[40, 0, 300], [129, 1, 7]], 264, 136
    L = Layer(counts, hidden)
    x, w, dh, pre = L.rows(hidden), L.weights(2 * inter, hidden), L.rows(inter), L.rows(2 * inter)

    def run(want_dx, want_dw):
        dpre, dx, dw = L.unwritten(2 * inter), L.unwritten(hidden), torch.full_like(w, 77)
        flmoe.fl_moe_expert_gated_backward(*L.at, inter, 1, x if want_dw else None, w if want_dx else None, pre, None, dh, dpre,
                                           dx if want_dx else None, dw if want_dw else None)
        return dpre, dx, dw
    both = run(True, True)
    for want_dx, want_dw in ((True, False), (False, True), (False, False)):
        dpre, dx, dw = run(want_dx, want_dw)
        assert torch.equal(dpre, both[0])
        assert torch.equal(dx, both[1]) if want_dx else bool((dx == 77).all())
        assert torch.equal(dw, both[2]) if want_dw else bool((dw == 77).all())


@pytest.mark.gpu
def test_calls_without_any_rows():
    """No expert has rows: rows are left as they are, weight gradients are zero."""
    in_, out = 384, 256
    L = Layer([[0, 0, 0], [0, 0, 0]], in_)
    x, w, dy = L.rows(in_), L.weights(out, in_), L.rows(out)
    y, dx, dw = L.unwritten(out), L.unwritten(in_), torch.full_like(w, 77)
    flmoe.fl_moe_expert_product(*L.at, in_, out, x, w, y)
    flmoe.fl_moe_expert_product_backward(*L.at, in_, out, x, w, dy, dx, dw)
    h, pre, dpre = L.unwritten(out // 2), L.unwritten(out), L.unwritten(out)
    flmoe.fl_moe_expert_gated(*L.at, out // 2, 0, x, w, h, pre)
    dv = torch.full_like(w, 77)
    flmoe.fl_moe_expert_gated_backward(*L.at, out // 2, 0, x, w, pre, None, L.rows(out // 2), dpre, dx, dv)
    (x8, xs), (w8, ws, _) = e4m3_rows(L, in_), e4m3_weights(L, out, in_)
    y8, h8, hs = L.unwritten(out), L.unwritten(out // 2, torch.uint8), L.unwritten(1, torch.float32)
    flmoe.fl_moe_expert_product_e4m3(*L.at, in_, out, x8, xs, w8, ws, y8)
    flmoe.fl_moe_expert_gated_e4m3(*L.at, out // 2, 1, x8, xs, w8, ws, h8, hs)
    for left in (y, dx, h, pre, dpre, y8, h8, hs):
        assert bool((left == 77).all())
    assert not bool(dw.any()) and not bool(dv.any())


@pytest.mark.gpu
def test_calls_on_several_streams_at_once():
    """The calls keep nothing and share nothing: three streams of them, of different sizes, run beside each other."""
    layers, streams = [], [torch.cuda.Stream() for _ in range(3)]
    for n, (counts, in_, out) in enumerate((([[300, 5], [40, 700]], 1024, 520), ([[16] * 16] * 2, 2056, 256), ([[1200]], 512, 1032))):
        L = Layer(counts, in_, seed=n)
        layers.append((L, in_, out, L.rows(in_), L.weights(out, in_), L.rows(out)))

    def run(stream, L, in_, out, x, w, dy, y, dx, dw):
        for _ in range(4):
            flmoe.fl_moe_expert_product(*L.at, in_, out, x, w, y, stream=stream)
            flmoe.fl_moe_expert_product_backward(*L.at, in_, out, x, w, dy, dx, dw, stream=stream)

    def results():
        return [(L.unwritten(out), L.unwritten(in_), torch.full_like(w, 77)) for L, in_, out, _, w, _ in layers]
    apart, together = results(), results()
    for given, got in zip(layers, apart):
        run(None, *given, *got)
    torch.cuda.synchronize()
    for _ in range(3):
        for stream, given, got in zip(streams, layers, together):
            run(stream, *given, *got)
    torch.cuda.synchronize()
    for one, other in zip(apart, together):
        for a, b in zip(one, other):
            assert torch.equal(a, b)
