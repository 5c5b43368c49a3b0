"""What the linear-attention entry points refuse, before any device work (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2002_03629_amd import binding as B

P = C.c_void_p(4096)       # a pointer that is never followed


def config(**kw):
    base = dict(B=2, T=8, heads=4, kv_heads=2, Dk=16, Dv=16, dtype=B.MADE_BF16, scale=1.0, ld_q=0, ld_k=0, ld_v=0, ld_o=0, offsets=None)
    base.update(kw)
    return B.linattn_config(*base.values())


def calls(cfg, q=P, ws=None, ws_bytes=0, ds_in=None, ds_out=None):
    L, n = B.lib(), None
    c = C.byref(cfg) if cfg is not None else None
    yield L.linattn_forward(c, q, P, P, P, n, P, n, ws, ws_bytes, n)
    yield L.linattn_backward(c, q, P, P, P, n, P, ds_out, P, P, P, ds_in, ws, ws_bytes, n)


BAD = [dict(B=-1), dict(Dk=0), dict(Dv=129), dict(heads=3), dict(kv_heads=0), dict(heads=0), dict(dtype=2), dict(scale=float("nan")),
       dict(scale=float("inf")), dict(ld_q=63), dict(ld_k=31), dict(ld_v=1), dict(ld_o=-5), dict(ld_q=1 << 24), dict(heads=1 << 20)]


@pytest.mark.parametrize("bad", BAD + [dict(T=-1)], ids=str)
def test_bad_sizes(bad):
    for code in calls(config(**bad)):
        assert code == B.MADE_ERR_ARG
        assert "linattn" in B.made_last_error()
    out = C.c_int64()
    assert B.lib().linattn_workspace_bytes(C.byref(config(**bad)), 0, C.byref(out)) == B.MADE_ERR_ARG


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_bad_sizes_of_a_step(bad):
    assert B.lib().linattn_step(C.byref(config(**bad)), P, P, P, P, P, 2, None, P, None) == B.MADE_ERR_ARG


def test_null_arguments_and_workspaces():
    assert all(code == B.MADE_ERR_ARG for code in calls(None))
    assert all(code == B.MADE_ERR_ARG for code in calls(config(), q=None))
    assert all(code == B.MADE_ERR_ARG for code in calls(config(), ws=C.c_void_p(4097), ws_bytes=1 << 20))
    L = B.lib()
    assert L.linattn_workspace_bytes(C.byref(config()), 0, None) == B.MADE_ERR_ARG
    assert list(calls(config(), ds_in=P, ds_out=P))[1] == B.MADE_ERR_ARG and "d_state" in B.made_last_error()
    assert L.linattn_step(C.byref(config()), P, P, P, P, None, 2, None, P, None) == B.MADE_ERR_ARG
    assert L.linattn_step(C.byref(config()), P, P, P, P, P, 1, None, P, None) == B.MADE_ERR_ARG      # fewer places than rows
    assert L.linattn_step(C.byref(config()), P, P, P, P, P, -1, P, P, None) == B.MADE_ERR_ARG


def refused(code, text):
    return code == B.MADE_ERR_ARG and text in B.made_last_error()


def test_more_than_a_launch_takes():
    """T beyond 2^30; workgroups of 2^32 threads together (bf16, widths of 128: 512 each; a step's have 256)"""
    L, q = B.lib(), [C.c_void_p(4096 * (i + 1)) for i in range(12)]
    out = C.c_int64()
    for T in ((1 << 30) + 1, (1 << 31) - 1):
        assert refused(L.linattn_workspace_bytes(C.byref(config(T=T)), 0, C.byref(out)), "T=")
        assert refused(L.linattn_forward(C.byref(config(T=T)), *q[:4], None, q[4], None, None, 0, None), "T=")
    assert L.linattn_workspace_bytes(C.byref(config(T=1 << 30)), 0, C.byref(out)) == B.MADE_OK and out.value > 0
    wide = config(B=1 << 23, T=1, heads=1, kv_heads=1, Dk=128, Dv=128)
    assert refused(L.linattn_forward(C.byref(wide), *q[:4], None, q[4], None, None, 0, None), "launch")
    wide.B = 3 << 20
    assert refused(L.linattn_backward(C.byref(wide), *q[:4], None, q[4], None, *q[5:8], None, None, 0, None), "launch")
    wide.B = 1 << 24
    assert refused(L.linattn_step(C.byref(wide), *q[:5], 1 << 24, None, q[5], None), "launch")


def test_an_output_that_is_an_input():
    L, q = B.lib(), [C.c_void_p(4096 * (i + 1)) for i in range(12)]
    for i in range(3):
        assert refused(L.linattn_forward(C.byref(config()), *q[:4], None, q[i], None, None, 0, None), "inputs")
        assert refused(L.linattn_step(C.byref(config()), *q[:5], 2, None, q[i], None), "inputs")
        for j in (0, 1, 2, 4):
            grads = q[5:8]
            grads[i] = q[j]
            assert refused(L.linattn_backward(C.byref(config()), *q[:4], None, q[4], None, *grads, None, None, 0, None), "inputs")
        grads = q[5:8]
        grads[i] = grads[i - 1]
        assert refused(L.linattn_backward(C.byref(config()), *q[:4], None, q[4], None, *grads, None, None, 0, None), "two gradients")


def test_states_workspaces_and_small_arrays_that_are_another_array():
    """every array a call writes against every other one, at its own address; a state alone may be replaced in place"""
    L, off = B.lib(), 4096 * 40
    cfg = config(T=5000, offsets=off)                                    # (long enough to be cut: the workspace is used)
    names = ["q", "k", "v", "log_decay", "state_in", "o", "state_out", "workspace"]
    back = ["q", "k", "v", "log_decay", "state_in", "d_o", "d_state_out", "dq", "dk", "dv", "d_state_in", "workspace"]
    step = ["q", "k", "v", "log_decay", "state", "slots", "o"]
    fresh = lambda ns: {n: 4096 * (i + 1) for i, n in enumerate(ns)}

    def forward(p):
        return L.linattn_forward(C.byref(cfg), *(p[n] for n in names), 1 << 30, None)

    def backward(p):
        return L.linattn_backward(C.byref(cfg), *(p[n] for n in back), 1 << 30, None)

    def one_step(p):
        return L.linattn_step(C.byref(cfg), *(p[n] for n in step[:5]), 2, p["slots"], p["o"], None)

    for call, ns, written in ((forward, names, ("o", "state_out", "workspace")), (one_step, step, ("state", "o")),
                              (backward, back, ("dq", "dk", "dv", "d_state_in", "workspace"))):
        for w in written:
            for other in ns:
                if other == w or (call is forward and {w, other} == {"state_in", "state_out"}):
                    continue
                p = fresh(ns)
                p[w] = p[other]
                assert call(p) == B.MADE_ERR_ARG, (w, other)
                assert any(x in B.made_last_error() for x in ("inputs", "one array", "d_state_out")), (w, other, B.made_last_error())
            if call is not one_step:
                assert call({**fresh(ns), w: off}) == B.MADE_ERR_ARG, w


def test_the_binding_refuses_other_types():
    with pytest.raises(ValueError, match="float16"):
        B.linattn_workspace_bytes(1, 64, 4, 2, 16, 16, torch.float16)


def test_the_binding_refuses_a_stream_of_another_device(monkeypatch):
    class Of:
        is_cuda = True

        def __init__(self, index):
            self.device = torch.device("cuda", index)

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    assert B._on_device(Of(0), "x") and B._on_device(Of(0), "x", Of(0))
    for t, s in ((1, None), (1, 0), (1, 1), (0, 1)):
        with pytest.raises(ValueError, match="cuda:1"):
            B._on_device(Of(t), "x", None if s is None else Of(s))


def test_a_prepared_step_refuses_another_current_device(monkeypatch):
    calls = []

    class Library:
        @staticmethod
        def linattn_step(*args):
            calls.append(args)
            return B.MADE_OK

    device = [None]                                                    # (tensors of the host, a library that computes nothing)
    monkeypatch.setattr(B, "_on_device", lambda t, *a: t)
    monkeypatch.setattr(B, "_stream", lambda s: None)
    monkeypatch.setattr(B, "lib", Library)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: device[0])
    x, state = torch.zeros(1, 2, 4), torch.zeros(1, 2, 4, 4)
    step = B.PreparedLinattnStep(x, x, x, torch.zeros(2), state, None, 1, 2, 2, 4, 4, 1.0, torch.zeros(1, 2, 4))
    step()
    device[0] = 1
    with pytest.raises(ValueError, match="cuda:1"):
        step()
    device[0] = None
    step()
    assert len(calls) == 2


def test_an_empty_batch_needs_no_pointers():
    L = B.lib()
    c = C.byref(config(B=0))
    assert L.linattn_forward(c, None, None, None, None, None, None, None, None, 0, None) == B.MADE_OK
    assert L.linattn_backward(c, *[None] * 12, 0, None) == B.MADE_OK
    assert L.linattn_step(c, None, None, None, None, None, 0, None, None, None) == B.MADE_OK


def test_workspace_sizes():
    one = B.linattn_workspace_bytes(1, 64, 4, 2, 16, 16, torch.bfloat16)
    assert one == 0                                            # one block: nothing to cut
    long_ = B.linattn_workspace_bytes(1, 30000, 4, 2, 16, 16, torch.bfloat16)
    assert long_ > 0 and long_ % (2 * 16 * 16 * 4) == 0
    assert B.linattn_workspace_bytes(1, 30000, 4, 2, 16, 16, torch.bfloat16, backward=True) > 0
    many = B.linattn_workspace_bytes(4096, 200, 8, 8, 128, 128, torch.bfloat16)
    assert many == 0                                           # the sequences alone fill the device
    with pytest.raises(B.MadeError):
        B.linattn_workspace_bytes(1, 64, 3, 2, 16, 16, torch.bfloat16)


def test_the_binding_refuses_tensors_of_the_host():
    x = torch.zeros(2, 8, 4, 16, dtype=torch.bfloat16)
    d = torch.zeros(4)
    with pytest.raises(ValueError, match="GPU"):
        B.linattn_forward(x, x, x, d, None, None, 2, 8, 4, 4, 16, 16, 1.0, x)
    with pytest.raises(ValueError):
        B.linattn_forward(x.half(), x, x, d, None, None, 2, 8, 4, 4, 16, 16, 1.0, x)
