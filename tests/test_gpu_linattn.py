"""GPU parity of the linear-attention entry points (include/jacobi_linattn.h) against oracle/linattn_oracle.py.

Tolerances are bounds of the arithmetic, element by element: A is the sum of the absolute values of an output's terms (the
oracle on absolute inputs).
  * fp32 sums: every term passes at most N roundings of 2^-24: a product's sum over D, a sum over a block of 64 steps, a
    block's or a segment's step of the state (two each), the factors lambda^n (their exponent's rounding counts |n log2
    lambda|, of which at most 150 before the factor is zero) and a handful of single ones.
  * bf16 operands of the second product (two parts each, of which this allows one): the scores, the decayed values and the
    state that is read are rounded once each, and no term meets more than two of these roundings: 2 x 2^-8 A; the output's
    rounding is 2^-8 of its value.
The states that leave a call are fp32 sums whatever the type of the steps.
"""
import numpy as np
import pytest
import torch

from oracle import linattn_oracle as L
from paper_2002_03629_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def rounded(g, shape, dtype, std=1.0):
    """normal values of the type, as a device tensor and as what they are in fp64"""
    t = torch.from_numpy(g.normal(size=shape).astype(np.float32) * np.float32(std)).to(DT[dtype])
    return t.cuda(), t.double().numpy()


def decays(kv, kind):
    if kind == "none":
        return np.zeros(kv, np.float32)
    if kind == "mixed":
        d = -np.exp2(-8.0 * np.arange(1, kv + 1) / kv)
        return d.astype(np.float32)
    if kind == "ends":        # no memory at all, an underflowing one, and none lost
        return np.resize(np.array([-np.inf, -200.0, 0.0, -1e-4], np.float32), kv)
    raise ValueError(kind)


class Case:
    def __init__(self, dtype, lengths, heads, kv, Dk, Dv, decay="mixed", packed=False, spare=0, carry=True, seed=0, wide=0, shift=0):
        self.dtype, self.lengths, self.heads, self.kv, self.Dk, self.Dv, self.packed = dtype, lengths, heads, kv, Dk, Dv, packed
        g = np.random.default_rng(seed)
        n = len(lengths)
        self.B = n
        self.T = sum(lengths) + spare if packed else lengths[0]
        assert packed or all(x == self.T for x in lengths)
        self.lead = (self.T,) if packed else (n, self.T)
        self.scale = float(np.float32(Dk ** -0.5))
        self.wide, self.shift = wide, shift
        self.t, self.x = {}, {}
        for key, h, D in (("q", heads, Dk), ("k", kv, Dk), ("v", kv, Dv), ("do", heads, Dv)):
            t, self.x[key] = rounded(g, self.lead + (h, D), dtype)
            self.t[key] = self.place(t)
        for key in ("s", "ds"):
            t, self.x[key] = rounded(g, (n, kv, Dk, Dv), "f32")
            self.t[key] = t
            if not carry:
                self.t[key], self.x[key] = None, np.zeros((n, kv, Dk, Dv))
        self.ld = decays(kv, decay)
        self.t["ld"] = torch.from_numpy(self.ld).cuda()
        self.offsets = None
        if packed:
            self.offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda()

    def place(self, t):
        """the tensor, or a copy whose rows lie `wide` elements further apart and begin `shift` elements into the memory"""
        if not self.wide and not self.shift:
            return t
        flat = t.reshape(-1, t.shape[-2] * t.shape[-1])
        buf = torch.full((flat.shape[0] * (flat.shape[1] + self.wide) + self.shift,), float("nan"), dtype=t.dtype, device="cuda")
        rows = buf[self.shift:].view(flat.shape[0], -1)[:, :flat.shape[1]]
        rows.copy_(flat)
        return rows.unflatten(1, t.shape[-2:]).unflatten(0, t.shape[:-2])

    def out(self, heads, D):
        return self.place(torch.full(self.lead + (heads, D), 7.0, dtype=DT[self.dtype], device="cuda"))

    def rows(self, b):
        if not self.packed:
            return (b, slice(0, self.T))
        at = sum(self.lengths[:b])
        return (slice(at, at + self.lengths[b]),)

    def spare(self, t):
        return t[sum(self.lengths):] if self.packed else t[:0]

    def roundings(self, n):
        g2 = np.abs(np.where(np.isfinite(self.ld), self.ld, 0)).max() * 1.45
        return self.Dk + self.Dv + 64 + 4 * (n // 32 + 1) + 2 * min(150.0, n * g2) + 16

    def sizes(self):
        return self.B, self.T, self.heads, self.kv, self.Dk, self.Dv, self.scale

    def oracle(self, fn, b, absolute=False):
        f = np.abs if absolute else (lambda a: a)
        x = [f(self.x[key][self.rows(b)]) for key in ("q", "k", "v", "do")]
        if fn == "forward":
            return L.forward(x[0], x[1], x[2], self.ld, self.scale, f(self.x["s"][b]))[:2]
        return L.backward(x[0], x[1], x[2], self.ld, self.scale, x[3], f(self.x["s"][b]), f(self.x["ds"][b]))

    def compare(self, fn, got):
        """got: outputs over steps, then the state"""
        for b in range(self.B):
            ref, mag = self.oracle(fn, b), self.oracle(fn, b, True)
            f32 = self.roundings(self.lengths[b]) * 2.0 ** -24
            for i, (r, m) in enumerate(zip(ref, mag)):
                steps = i < len(ref) - 1
                if got[i] is None:
                    continue
                y = (got[i][self.rows(b)] if steps else got[i][b]).double().cpu().numpy()
                tol = f32 * m + 1e-37
                if steps and self.dtype == "bf16":
                    tol = tol + 2 * 2.0 ** -8 * m + 2.0 ** -8 * np.abs(r)
                bad = ~(np.abs(y - r) <= tol)
                assert not bad.any(), (fn, i, b, int(bad.sum()), y[bad][:4], r[bad][:4], tol[bad][:4])

    def forward(self, workspace=None, o=None, state_out="new", state_in="given"):
        o = self.out(self.heads, self.Dv) if o is None else o
        s_in = self.t["s"] if isinstance(state_in, str) else state_in
        if isinstance(state_out, str):
            state_out = torch.full((self.B, self.kv, self.Dk, self.Dv), 7.0, device="cuda")
        B.linattn_forward(self.t["q"], self.t["k"], self.t["v"], self.t["ld"], s_in, self.offsets, *self.sizes(), o, state_out,
                          workspace=workspace)
        return o, state_out

    def backward(self, workspace=None, d_state=True):
        outs = [self.out(self.heads, self.Dk), self.out(self.kv, self.Dk), self.out(self.kv, self.Dv)]
        ds = torch.full((self.B, self.kv, self.Dk, self.Dv), 7.0, device="cuda") if d_state else None
        B.linattn_backward(self.t["q"], self.t["k"], self.t["v"], self.t["ld"], self.t["s"], self.offsets, self.t["do"],
                           self.t["ds"], *self.sizes(), *outs, ds, workspace=workspace)
        return outs + [ds]

    def check_all(self, workspace=None):
        got = self.forward(workspace)
        self.compare("forward", got)
        assert (self.spare(got[0]) == 7).all()
        got = self.backward(workspace)
        self.compare("backward", got)
        for g in got[:3]:
            assert (self.spare(g) == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 63, 64, 65, 127, 129, 200])
def test_lengths(dtype, T):
    Case(dtype, [T] * 2, 4, 2, 64, 32, seed=T).check_all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Dk,Dv", [(1, 1), (7, 128), (128, 3), (32, 64), (64, 128), (128, 32), (20, 33), (72, 100), (128, 128), (96, 40)])
def test_widths(dtype, Dk, Dv):
    Case(dtype, [150], 3, 3, Dk, Dv, seed=Dk).check_all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 1), (6, 2), (5, 5), (12, 4), (16, 1), (9, 3)])
def test_shared_states(dtype, heads, kv):
    Case(dtype, [100] * 3, heads, kv, 32, 64, seed=heads).check_all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("decay", ["none", "ends"])
def test_decays(dtype, decay):
    Case(dtype, [180], 4, 4, 32, 32, decay=decay).check_all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths", [[5, 0, 1, 130, 64], [0], [0, 0, 3], [300, 2] + [1] * 70 + [90, 0], [65] * 9])
def test_packed(dtype, lengths):
    Case(dtype, lengths, 4, 2, 32, 64, packed=True, spare=3).check_all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_steps(dtype):
    """sequences of no steps hand their states on"""
    c = Case(dtype, [0] * 3, 4, 2, 64, 32)
    o, s = c.forward()
    assert o.numel() == 0 and torch.equal(s, c.t["s"])
    *_, ds = c.backward()
    assert torch.equal(ds, c.t["ds"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e-20, 1e25])
def test_values_far_from_one(dtype, size):
    c = Case(dtype, [200], 2, 2, 64, 64, decay="none")
    for key in ("v", "s"):
        c.t[key] = (c.t[key].double() * size).to(c.t[key].dtype)
        c.x[key] = c.t[key].double().cpu().numpy()
    c.compare("forward", c.forward())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bf16_outputs_are_off_by_little_more_than_their_own_rounding(dtype):
    """Scores, states and decayed values are two bf16 parts each: 2^-17 of every term, three roundings at most, beside fp32's
    (a bound 1.5 % above that of the output's rounding alone where A is of the output's size)."""
    for heads, kv, decay in ((2, 2, "mixed"), (4, 1, "none")):
        c = Case(dtype, [500], heads, kv, 128, 128, decay=decay, carry=False)
        o, _ = c.forward(state_out=None)
        ref, mag = c.oracle("forward", 0)[0], c.oracle("forward", 0, True)[0]
        err = np.abs(o[0].double().cpu().numpy() - ref)
        tol = c.roundings(500) * 2.0 ** -24 * mag
        if dtype == "bf16":
            tol = tol + 3 * 2.0 ** -17 * mag + 2.0 ** -8 * np.abs(ref)
        assert (err <= tol).all()


@pytest.mark.parametrize("decay", ["mixed", "none"])
@pytest.mark.parametrize("lengths,heads,kv,Dk,Dv,packed", [([300], 2, 2, 128, 128, False), ([1100], 4, 1, 128, 64, False), ([90, 90], 6, 2, 40, 72, False),
                                                           ([700, 3, 0, 450, 64], 4, 2, 64, 96, True)])
def test_bf16_outputs_and_gradients_with_states(lengths, heads, kv, Dk, Dv, packed, decay):
    """As above, for gradients too, with states that enter and their gradients, cut and whole.  A term that reaches an output through a
    block's scores is rounded to two bf16 parts once; one that reaches it through the state twice: as a decayed value and where the
    state is read (whose value a segment's sum and the state that enters have their share in).  Each is off by 2^-17 of the
    term at most: a part's rounding is half a step of 2^-7, the first one's rest is below 2^-8 of the value, a half step of it
    2^-8 of that, and of the rest's own binade half again."""
    c = Case("bf16", lengths, heads, kv, Dk, Dv, decay=decay, packed=packed, spare=2 if packed else 0, seed=heads)
    for fn in ("forward", "backward"):
        for n in (1 << 24, 256):
            got = getattr(c, fn)(workspace=torch.empty(n, dtype=torch.uint8, device="cuda"))
            for b in range(c.B):
                ref, mag = c.oracle(fn, b), c.oracle(fn, b, True)
                for i in range(len(ref) - 1):
                    err = np.abs(got[i][c.rows(b)].double().cpu().numpy() - ref[i])
                    tol = (c.roundings(lengths[b]) * 2.0 ** -24 + 3 * 2.0 ** -17) * mag[i] + 2.0 ** -8 * np.abs(ref[i])
                    assert (err <= tol).all(), (fn, n, b, i, (err / tol).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_carried_state(dtype):
    c = Case(dtype, [140] * 2, 2, 2, 64, 64, carry=False)
    o, s = c.forward(state_out=None)
    c.compare("forward", (o, s))
    c.compare("backward", c.backward(d_state=False))
    c.check_all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("wide,shift", [(64, 0), (24, 8), (3, 0), (0, 1), (5, 3)])
def test_rows_apart_and_unaligned(dtype, wide, shift):
    for packed in (False, True):
        Case(dtype, [90, 90], 2, 1, 40, 48, wide=wide, shift=shift, packed=packed).check_all()


def test_parts_of_one_projection():
    """q, k and v as parts of one tensor, their gradients as parts of another"""
    c = Case("bf16", [130] * 2, 4, 4, 64, 64)
    qkv = torch.cat([c.t[x] for x in "qkv"], dim=2)
    assert qkv.shape == (2, 130, 12, 64)
    c.t["q"], c.t["k"], c.t["v"] = qkv[:, :, :4], qkv[:, :, 4:8], qkv[:, :, 8:]
    c.compare("forward", c.forward())
    d = torch.full_like(qkv, 7.0)
    parts = [d[:, :, :4], d[:, :, 4:8], d[:, :, 8:]]
    B.linattn_backward(c.t["q"], c.t["k"], c.t["v"], c.t["ld"], c.t["s"], None, c.t["do"], c.t["ds"], *c.sizes(), *parts)
    c.compare("backward", parts + [None])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_sequences_cut_and_whole(dtype):
    """with a workspace the sequences are cut into segments; with one that is too small they are not"""
    for c in (Case(dtype, [1100], 2, 2, 64, 96), Case(dtype, [700, 3, 0, 450], 4, 2, 128, 64, packed=True, spare=2)):
        for back in (False, True):
            need = B.linattn_workspace_bytes(c.B, c.T, c.heads, c.kv, c.Dk, c.Dv, DT[dtype], packed=c.packed, backward=back)
            assert need > 0
            run = c.backward if back else c.forward
            for n in (need, 256):
                ws = torch.full((n + 256,), 255, dtype=torch.uint8, device="cuda")
                c.compare("backward" if back else "forward", run(workspace=ws[:n]))
                assert (ws[n:] == 255).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,B_", [(1, 3), (200, 2), (1000, 1)])
def test_state_in_place(dtype, T, B_):
    c = Case(dtype, [T] * B_, 6, 2, 64, 64)
    ref = c.forward()
    state = c.t["s"].clone()
    o, _ = c.forward(state_in=state, state_out=state)
    assert torch.equal(o, ref[0]) and torch.equal(state, ref[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv,D", [(8, 1, 128), (6, 2, 64)])
def test_packed_states_in_place(dtype, heads, kv, D):
    """sequences of one segment and of several, where workgroups share a state's query heads: as with a state for the result"""
    c = Case(dtype, [1, 0, 64, 700, 30, 1300, 5], heads, kv, D, D, packed=True, spare=2)
    assert B.linattn_workspace_bytes(c.B, c.T, heads, kv, D, D, DT[dtype], packed=True) > 0
    ref = c.forward()
    c.compare("forward", ref)
    for _ in range(3):
        state = c.t["s"].clone()
        o, _ = c.forward(state_in=state, state_out=state)
        assert torch.equal(o, ref[0]) and torch.equal(state, ref[1])


def test_equal_calls_give_equal_bits():
    c = Case("bf16", [900] * 2, 8, 2, 128, 128)
    a, b = c.backward(), c.backward()
    assert all(torch.equal(x, y) for x, y in zip(a, b))


# ---------------------------------------------------------------------------------------------------------- single steps
def step_oracle(q, k, v, ld, scale, state, slots):
    o = {}
    state = state.copy()
    for r, s in enumerate(slots):
        if 0 <= s < len(state):
            y, end, _ = L.forward(q[r:r + 1], k[r:r + 1], v[r:r + 1], ld, scale, state[s])
            state[s] = end
            o[r] = y[0]
    return o, state


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,slots", [(1, None), (3, None), (5, [4, -1, 0, 9, 2]), (7, [1, 1, 3, 1, -1, 3, 0]), (300, "many")])
@pytest.mark.parametrize("heads,kv,Dk,Dv", [(4, 2, 64, 64), (10, 1, 128, 128), (3, 3, 17, 30), (2, 2, 1, 1), (4, 4, 100, 72)])
def test_step(dtype, n, slots, heads, kv, Dk, Dv):
    g = np.random.default_rng(n + heads)
    pool = 9 if n < 10 else 310
    if slots == "many":
        slots = g.permutation(pool)[:n]
        slots[5], slots[200], slots[299] = slots[250], slots[250], -3
    place = np.arange(n) if slots is None else np.asarray(slots)
    (q, q64), (k, k64), (v, v64) = (rounded(g, (n, h, D), dtype) for h, D in ((heads, Dk), (kv, Dk), (kv, Dv)))
    state, s64 = rounded(g, (pool, kv, Dk, Dv), "f32")
    ld = decays(kv, "mixed")
    scale = float(np.float32(Dk ** -0.5))
    o = torch.full((n, heads, Dv), 7.0, dtype=DT[dtype], device="cuda")
    d_slots = None if slots is None else torch.from_numpy(place.astype(np.int32)).cuda()
    B.linattn_step(q, k, v, torch.from_numpy(ld).cuda(), state, d_slots, n, heads, kv, Dk, Dv, scale, o)
    ref, s_ref = step_oracle(q64, k64, v64, ld, scale, s64, place)
    mag, s_mag = step_oracle(*(np.abs(x) for x in (q64, k64, v64)), ld, scale, np.abs(s64), place)
    # a state's element takes a product, a product and sum, and lambda (3 roundings) for each row that names it
    same = max(np.bincount(place[place >= 0])) if (place >= 0).any() else 1
    tol = (5 * same) * 2.0 ** -24
    assert (np.abs(state.double().cpu().numpy() - s_ref) <= tol * s_mag).all()
    got = o.double().cpu().numpy()
    for r in range(n):
        if r not in ref:
            assert (got[r] == 7).all()
            continue
        t = (5 * same + Dk + 8) * 2.0 ** -24 * mag[r] + (2.0 ** -8 * np.abs(ref[r]) if dtype == "bf16" else 0)
        assert (np.abs(got[r] - ref[r]) <= t).all(), r


def test_step_on_parts_and_odd_memory():
    """rows apart and unaligned (also the state's)"""
    g = np.random.default_rng(1)
    n, heads, kv, D = 5, 4, 2, 36
    qkv, x64 = rounded(g, (n, 8, D), "bf16")
    q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    buf = torch.zeros(n * kv * D * D + 1, device="cuda")
    state = buf[1:].view(n, kv, D, D)
    o = torch.zeros(n, 4, D, dtype=torch.bfloat16, device="cuda")
    ld = decays(kv, "mixed")
    B.linattn_step(q, k, v, torch.from_numpy(ld).cuda(), state, None, n, heads, kv, D, D, 0.5, o)
    ref, s_ref = step_oracle(x64[:, :4], x64[:, 4:6], x64[:, 6:], ld, 0.5, np.zeros((n, kv, D, D)), np.arange(n))
    mag, _ = step_oracle(*(np.abs(x64[:, a:b]) for a, b in ((0, 4), (4, 6), (6, 8))), ld, 0.5, np.zeros((n, kv, D, D)), np.arange(n))
    assert (np.abs(state.double().cpu().numpy() - s_ref) <= 3 * 2.0 ** -24 * np.abs(s_ref)).all()
    for r in range(n):
        assert (np.abs(o[r].double().cpu().numpy() - ref[r]) <= (D + 12) * 2.0 ** -24 * mag[r] + 2.0 ** -8 * np.abs(ref[r])).all()


# ------------------------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_then_single_steps(dtype):
    """a prompt of 70 steps into a pool's state, then 5 steps one by one: as 75 steps at once"""
    c = Case(dtype, [75], 4, 2, 64, 48)
    whole, end = c.forward()
    c.compare("forward", (whole, end))
    cut = Case(dtype, [70], 4, 2, 64, 48)
    cut.t = dict(c.t)
    cut.t["q"], cut.t["k"], cut.t["v"] = (c.t[x][:, :70].contiguous() for x in "qkv")
    pool = torch.zeros(3, 2, 64, 48, device="cuda")
    o, _ = cut.forward(state_out=pool[1:2])
    slots = torch.tensor([1], dtype=torch.int32, device="cuda")
    outs = [o]
    for t in range(70, 75):
        y = torch.empty(1, 4, 48, dtype=DT[dtype], device="cuda")
        B.linattn_step(*(c.t[x][:, t] for x in "qkv"), c.t["ld"], pool, slots, 1, 4, 2, 64, 48, c.scale, y)
        outs.append(y[:, None])
    c.compare("forward", (torch.cat(outs, 1), pool[1:2]))
    assert (pool[0] == 0).all() and (pool[2] == 0).all()


@pytest.mark.parametrize("dtype,T", [("bf16", 300), ("f32", 150)])
def test_rows_as_far_apart_as_they_may_be(dtype, T):
    """2^23 elements from row to row: the last rows lie beyond 4 GiB, a block spans 1 GiB"""
    c = Case(dtype, [T], 2, 2, 32, 32, wide=(1 << 23) - 64)
    assert c.t["q"].stride(1) == 1 << 23 and c.t["q"].stride(1) * c.t["q"].element_size() * (T - 1) > 1 << 32
    c.compare("forward", c.forward())
    c.compare("backward", c.backward())
    torch.cuda.empty_cache()


def test_states_beyond_4_gib():
    n, g = 70000, np.random.default_rng(5)
    state = torch.zeros(n, 1, 128, 128, device="cuda")
    slots = torch.tensor([n - 1, 3, n - 2, n - 1], dtype=torch.int32, device="cuda")
    s0 = torch.from_numpy(g.normal(size=(3, 1, 128, 128)).astype(np.float32)).cuda()
    places = [n - 1, 3, n - 2]
    state[places] = s0
    q, k, v = (torch.from_numpy(g.normal(size=(4, 1, 128)).astype(np.float32)).cuda() for _ in range(3))
    ld, o, near, o2 = torch.full((1,), -0.1, device="cuda"), torch.empty_like(q), s0.clone(), torch.empty_like(q)
    B.linattn_step(q, k, v, ld, state, slots, 4, 1, 1, 128, 128, 0.1, o)
    B.linattn_step(q, k, v, ld, near, torch.tensor([0, 1, 2, 0], dtype=torch.int32, device="cuda"), 4, 1, 1, 128, 128, 0.1, o2)
    assert torch.equal(o, o2) and torch.equal(state[places], near)
    state[places] = 0
    assert not state.any()
    del state
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_sequences_than_a_cut_call_may_have(dtype):
    """one block each: the last ones are the same as in a call of their own"""
    n, T = 30000, 3
    c = Case(dtype, [T] * n, 2, 1, 16, 16)
    last = Case(dtype, [T] * 5, 2, 1, 16, 16)
    for key in ("q", "k", "v", "do", "s", "ds"):
        last.t[key].copy_(c.t[key][-5:])
        last.x[key] = c.x[key][-5:]
    for fn in ("forward", "backward"):
        all_, few = getattr(c, fn)(), getattr(last, fn)()
        last.compare(fn, few)
        last.compare(fn, [x[-5:] for x in all_])


@pytest.mark.parametrize("dtype,B_", [("f32", 34000), ("bf16", 70000)])
def test_more_packed_sequences_than_one_join_takes(dtype, B_):
    """a few long sequences, which are cut, among very many of a step or none; in gradients 68000 and 140000 pairs of a state and a
    role.  The long ones and the ends are those of a call of their own, the others those of an uncut call."""
    lengths = [(i * 7919) % 3 % 2 for i in range(B_)]
    long_ = {0: 400, 21846: 333, 33000: 1000, B_ - 1: 500}
    for b, n in long_.items():
        lengths[b] = n
    c = Case(dtype, lengths, 2, 1, 16, 16, packed=True, spare=3)
    only = sorted([*long_, 1, 21845, 32999, B_ - 2])
    at = np.concatenate([[0], np.cumsum(lengths)])
    rows = np.concatenate([np.arange(at[b], at[b + 1]) for b in only])
    few = Case(dtype, [lengths[b] for b in only], 2, 1, 16, 16, packed=True)
    for key in ("q", "k", "v", "do", "s", "ds"):
        pick = only if key in ("s", "ds") else rows
        few.t[key].copy_(c.t[key][pick])
        few.x[key] = c.x[key][pick]
    short = np.setdiff1d(np.arange(at[-1]), np.concatenate([np.arange(at[b], at[b + 1]) for b in long_]))
    for fn, back in (("forward", False), ("backward", True)):
        need = B.linattn_workspace_bytes(c.B, c.T, 2, 1, 16, 16, DT[dtype], packed=True, backward=back)
        assert need > 0
        cut = getattr(c, fn)(torch.empty(need, dtype=torch.uint8, device="cuda"))
        whole = getattr(c, fn)(torch.empty(256, dtype=torch.uint8, device="cuda"))
        few.compare(fn, [x[rows] for x in cut[:-1]] + [cut[-1][only]])
        for x, y in zip(cut[:-1], whole[:-1]):
            assert torch.equal(x[short], y[short]) and (c.spare(x) == 7).all()
        others = np.setdiff1d(np.arange(B_), list(long_))
        assert torch.equal(cut[-1][others], whole[-1][others])


@pytest.mark.parametrize("cut", [False, True])
def test_a_million_packed_sequences(cut):
    """of a step or none, one long sequence among them: in a time that does not grow with the square of their number"""
    n, D, g = 1 << 20, 8, np.random.default_rng(2)
    lengths = g.integers(0, 2, n)
    lengths[n // 2] = 300
    at = np.concatenate([[0], np.cumsum(lengths)])
    T, i = int(at[-1]), int(at[n // 2])
    q, k, v = (torch.from_numpy(g.normal(size=(T, 1, D)).astype(np.float32)).cuda() for _ in range(3))
    ld, offsets = torch.full((1,), -0.1, device="cuda"), torch.from_numpy(at.astype(np.int32)).cuda()
    need = B.linattn_workspace_bytes(n, T, 1, 1, D, D, torch.float32, packed=True) if cut else 256
    ws, o, end = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty_like(v), torch.empty(n, 1, D, D, device="cuda")
    B.linattn_forward(q, k, v, ld, None, offsets, n, T, 1, 1, D, D, 0.5, o, end, workspace=ws)
    q, k, v, o, end = (x.double().cpu().numpy()[:, 0] for x in (q, k, v, o, end))
    # a step alone: 8 products and sums, a factor; the state after it is the product
    one = np.setdiff1d(np.arange(T), np.arange(i, i + 300))
    ref, mag = 0.5 * (q * k).sum(1, keepdims=True) * v, 0.5 * np.abs(q * k).sum(1, keepdims=True) * np.abs(v)
    assert (np.abs(o - ref) <= 24 * 2.0 ** -24 * mag)[one].all()
    whose = np.repeat(np.arange(n), lengths)[one]
    assert (np.abs(end[whose] - k[one][:, :, None] * v[one][:, None, :]) <= 2 * 2.0 ** -24 * np.abs(end[whose])).all()
    assert not end[lengths == 0].any()
    ref, last, _ = L.forward(*(x[i:i + 300, None] for x in (q, k, v)), np.array([np.float32(-0.1)]), 0.5)
    mag, m_last, _ = L.forward(*(np.abs(x[i:i + 300, None]) for x in (q, k, v)), np.array([np.float32(-0.1)]), 0.5)
    tol = (2 * D + 64 + 4 * 10 + 2 * 45 + 16) * 2.0 ** -24
    assert (np.abs(o[i:i + 300] - ref[:, 0]) <= tol * mag[:, 0]).all() and (np.abs(end[n // 2] - last[0]) <= tol * m_last[0]).all()


def test_two_calls_at_once():
    """on two streams, a workspace each"""
    c = [Case("bf16", [3000], 4, 2, 64, 64, seed=i) for i in range(2)]
    ref = [(x.forward(), x.backward()) for x in c]
    need = [B.linattn_workspace_bytes(1, 3000, 4, 2, 64, 64, torch.bfloat16, backward=b) for b in (False, True)]
    assert min(need) > 0
    streams = [torch.cuda.Stream() for _ in c]
    ws = [[torch.empty(n, dtype=torch.uint8, device="cuda") for n in need] for _ in c]
    torch.cuda.synchronize()
    got = [None] * 2
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = (c[i].forward(workspace=ws[i][0]), c[i].backward(workspace=ws[i][1]))
    torch.cuda.synchronize()
    for i in range(2):
        for a, b in zip(ref[i], got[i]):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_captured_and_replayed():
    """forward, backward and a step in one graph, replayed on new inputs with eager work between"""
    c = Case("bf16", [400] * 2, 4, 2, 64, 64)
    fw = torch.empty(max(B.linattn_workspace_bytes(2, 400, 4, 2, 64, 64, torch.bfloat16), 256), dtype=torch.uint8, device="cuda")
    bw = torch.empty(max(B.linattn_workspace_bytes(2, 400, 4, 2, 64, 64, torch.bfloat16, backward=True), 256), dtype=torch.uint8, device="cuda")
    o, grads = c.out(4, 64), [c.out(4, 64), c.out(2, 64), c.out(2, 64)]
    s_out, ds = torch.empty(2, 2, 64, 64, device="cuda"), torch.empty(2, 2, 64, 64, device="cuda")
    y = torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda")

    def call(o, s_out, grads, ds, y, fw, bw):
        B.linattn_forward(c.t["q"], c.t["k"], c.t["v"], c.t["ld"], c.t["s"], None, *c.sizes(), o, s_out, workspace=fw)
        B.linattn_backward(c.t["q"], c.t["k"], c.t["v"], c.t["ld"], c.t["s"], None, c.t["do"], c.t["ds"], *c.sizes(), *grads, ds, workspace=bw)
        B.linattn_step(*(c.t[x][:, 0] for x in "qkv"), c.t["ld"], s_out, None, 2, 4, 2, 64, 64, c.scale, y)

    call(o, s_out, grads, ds, y, fw, bw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(o, s_out, grads, ds, y, fw, bw)
    for rep in range(4):
        for x in ("q", "k", "v", "do", "s", "ds"):
            c.t[x].copy_(torch.randn_like(c.t[x]))
        graph.replay()
        torch.cuda.synchronize()
        e = [torch.empty_like(o), torch.empty_like(s_out), [torch.empty_like(g) for g in grads], torch.empty_like(ds), torch.empty_like(y)]
        call(*e, None, None)
        torch.cuda.synchronize()
        for a, b in zip([o, s_out, ds, y] + grads, [e[0], e[1], e[3], e[4]] + e[2]):
            assert torch.equal(a, b), rep


def test_on_another_stream():
    c = Case("bf16", [500], 4, 4, 64, 64)
    ref = c.forward()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o, s = torch.empty_like(ref[0]), torch.empty_like(ref[1])
    for _ in range(3):
        B.linattn_forward(c.t["q"], c.t["k"], c.t["v"], c.t["ld"], c.t["s"], None, *c.sizes(), o, s, stream=side)
    side.synchronize()
    assert torch.equal(o, ref[0]) and torch.equal(s, ref[1])
