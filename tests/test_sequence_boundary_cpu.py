"""Refusals of the sequence operators' entry points: argument errors are reported before any GPU work, so this runs without a GPU."""
import ctypes

import pytest

import paper_1910_10892_amd as mrf
from paper_1910_10892_amd import mrfmp as binding

FAKE = 0x1000      # never dereferenced by the host checks
INF, NAN = float("inf"), float("nan")


def _attention(**given):
    c = binding._CAttention()
    values = dict(B=2, Q=40, K=50, Hq=4, Hk=2, D=16, type=0, scale=0.25, q=FAKE, k=FAKE, v=FAKE, first_offset=-(1 << 63), last_offset=(1 << 63) - 1)
    values.update(given)
    for name, value in values.items():
        setattr(c, name, (ctypes.c_int64 * 3)(*value) if name.endswith("stride") else value)
    return c


def test_attention_refusals():
    lib = mrf.load_library()

    def forward(out=FAKE, ws=FAKE, size=1 << 40, **given):
        return lib.mrf_attention_forward(ctypes.byref(_attention(**given)), out, None, ws, size, None)

    assert lib.mrf_attention_forward(None, FAKE, None, FAKE, 1 << 40, None) == -1
    for bad in (dict(B=-1), dict(Q=-1), dict(K=-1), dict(Hq=0), dict(Hk=0), dict(Hk=3), dict(D=0), dict(D=129), dict(Q=0x7fff0001),
                dict(B=1 << 20, Q=1 << 20), dict(B=1 << 20, K=1 << 20), dict(Hq=65538, Hk=2), dict(Q=1 << 30, K=0x3fff0001), dict(B=1 << 22), dict(B=1 << 14, Q=32769)):
        assert forward(**bad) == -2, bad
        assert lib.mrf_attention_workspace_bytes(ctypes.byref(_attention(**bad)), 1) == 0
    for bad in (dict(type=3), dict(type=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=INF), dict(scale=NAN), dict(scale=3e38), dict(q_stride=(1, -1, 1)),
                dict(k_stride=(-1, 1, 1)), dict(v_stride=(1, 1, -1)), dict(query_offset=1 << 41), dict(query_offset=-(1 << 41))):
        assert forward(**bad) == -12, bad
    table = dict(table=FAKE, bucket_of=FAKE, n_offsets=9, n_buckets=4)
    assert forward(**{**table, "n_buckets": 0}) == -2 and forward(**{**table, "n_buckets": 65537}) == -2
    for bad in (dict(n_offsets=0), dict(n_offsets=(1 << 40) + 1), dict(map_offset=(1 << 41) + 1), dict(map_offset=-(1 << 41) - 1)):
        assert forward(**{**table, **bad}) == -12, bad
    assert forward(**{**table, "bucket_of": None}) == -1
    for name in ("q", "k", "v"):
        assert forward(**{name: None}) == -1
    assert forward(out=None) == -1
    # nothing to do
    assert forward(B=0, q=None, k=None, v=None, out=None) == 0 and forward(Q=0, q=None, out=None) == 0
    # keys divided among workgroups need room for their parts
    row = dict(Q=1, K=4096)
    need = lib.mrf_attention_workspace_bytes(ctypes.byref(_attention(**row)), 0)
    assert need > 0 and lib.mrf_attention_workspace_bytes(ctypes.byref(_attention()), 0) == 0
    assert forward(ws=None, **row) == -1 and forward(size=need - 1, **row) == -6


def test_attention_backward_refusals():
    lib = mrf.load_library()
    need = lib.mrf_attention_workspace_bytes(ctypes.byref(_attention()), 1)
    assert need > 0

    def backward(g=FAKE, out=FAKE, lse=FAKE, gt=None, ws=FAKE, size=need, **given):
        return lib.mrf_attention_backward(ctypes.byref(_attention(**given)), g, out, lse, FAKE, FAKE, FAKE, gt, ws, size, None)

    assert backward(g=None) == -1 and backward(out=None) == -1 and backward(lse=None) == -1 and backward(ws=None) == -1
    assert backward(q=None) == -1 and backward(k=None) == -1 and backward(v=None) == -1 and backward(size=need - 1) == -6
    assert backward(gt=FAKE) == -1                      # a gradient of no table
    assert backward(D=0) == -2 and backward(type=7) == -12
    table = _attention(table=FAKE, bucket_of=FAKE, n_offsets=9, n_buckets=4)
    assert lib.mrf_attention_workspace_bytes(ctypes.byref(table), 1) > need


def _rotation(**given):
    c = binding._CHeadRotation()
    values = dict(B=2, T=3, Hq=4, Hk=2, D=16, type=0, q=FAKE, k=FAKE, eps=1e-6, rotary=16, inv_freq=FAKE, n_axes=1)
    values.update(given)
    for name, value in values.items():
        setattr(c, name, (ctypes.c_int64 * 3)(*value) if name.endswith("stride") else value)
    return c


def test_head_rotation_refusals():
    lib = mrf.load_library()

    def forward(out_q=FAKE, out_k=FAKE, **given):
        return lib.mrf_head_rotation_forward(bytes(_rotation(**given)), out_q, out_k, None)

    assert lib.mrf_head_rotation_forward(None, FAKE, FAKE, None) == -1
    for bad in (dict(B=-1), dict(T=-1), dict(Hq=-1), dict(Hk=-1), dict(D=0), dict(D=513), dict(B=1 << 16, T=1 << 16), dict(Hq=65537)):
        assert forward(**bad) == -2, bad
    for bad in (dict(type=3), dict(eps=0.0), dict(eps=-1.0), dict(eps=INF), dict(eps=NAN), dict(rotary=-2), dict(rotary=18), dict(rotary=7), dict(n_axes=0),
                dict(n_axes=3, positions=FAKE), dict(position_offset=1 << 41), dict(position_offset=-(1 << 41)), dict(q_stride=(1, 1, -1)), dict(k_stride=(-1, 1, 1))):
        assert forward(**bad) == -12, bad
    assert forward(n_axes=2) == -1 and forward(q=None) == -1 and forward(k=None) == -1 and forward(inv_freq=None) == -1
    assert forward(out_q=None) == -1 and forward(out_k=None) == -1
    assert forward(B=0, q=None, k=None, out_q=None, out_k=None) == 0 and forward(Hq=0, Hk=0, out_q=None, out_k=None) == 0

    need = mrf.mrf_head_rotation_workspace_bytes(6, 4, 2, 16)
    assert need > 0 and mrf.mrf_head_rotation_workspace_bytes(-1, 4, 2, 16) == 0 and mrf.mrf_head_rotation_workspace_bytes(6, 4, 2, 513) == 0

    def backward(gq=FAKE, gk=FAKE, gg=FAKE, ws=FAKE, size=need, **given):
        return lib.mrf_head_rotation_backward(bytes(_rotation(**given)), gq, gk, FAKE, FAKE, gg, None, ws, size, None)

    assert backward(gq=None) == -1 and backward(gk=None) == -1 and backward(ws=None) == -1 and backward(size=need - 1) == -6
    assert backward(D=0) == -2 and backward(type=-1) == -12
    assert backward(B=0, gq=None, gk=None, gg=None, ws=None, size=0) == 0


def test_gated_scan_refusals():
    lib = mrf.load_library()

    def forward(outer=2, T=3, inner=4, t=0, x=FAKE, xs=None, z=FAKE, zs=None, y=FAKE, ws=FAKE, size=1 << 40):
        strides = lambda s: None if s is None else (ctypes.c_int64 * 2)(*s)  # noqa: E731
        return lib.mrf_gated_scan_forward(outer, T, inner, t, x, strides(xs), z, strides(zs), 1, 0, None, None, y, None, None, ws, size, None)

    for bad in (dict(outer=-1), dict(T=-1), dict(inner=-1), dict(T=1 << 31), dict(outer=1 << 31), dict(inner=1 << 31), dict(outer=1 << 20, inner=1 << 20), dict(outer=2, inner=1 << 30)):
        assert forward(**bad) == -2, bad
        assert mrf.mrf_gated_scan_workspace_bytes(bad.get("outer", 2), bad.get("T", 3), bad.get("inner", 4)) == 0
    assert forward(t=3) == -12 and forward(xs=(-1, 4)) == -12 and forward(zs=(12, -4)) == -12
    assert forward(x=None) == -1 and forward(z=None) == -1 and forward(y=None) == -1
    assert forward(outer=0, x=None, z=None, y=None) == 0 and forward(inner=0, x=None, z=None, y=None) == 0
    need = mrf.mrf_gated_scan_workspace_bytes(2, 5000, 4)
    assert need > 0 and mrf.mrf_gated_scan_workspace_bytes(2, 3, 4) == 0
    assert forward(T=5000, ws=None) == -1 and forward(T=5000, size=need - 1) == -6
    assert mrf.mrf_gated_scan_states(0) == 0 and mrf.mrf_gated_scan_states(1) == 1 and mrf.mrf_gated_scan_states(-5) == 0
    assert 16 * mrf.mrf_gated_scan_states(1000) >= 1000

    def backward(gy=FAKE, states=FAKE, x=FAKE, ws=FAKE, size=need):
        return lib.mrf_gated_scan_backward(2, 5000, 4, 0, gy, None, x, None, FAKE, None, 1, 0, None, states, FAKE, FAKE, None, ws, size, None)

    assert backward(gy=None) == -1 and backward(states=None) == -1 and backward(x=None) == -1 and backward(ws=None) == -1 and backward(size=need - 1) == -6


def test_bindings_refuse_tensors_that_do_not_fit():
    import torch
    q, k = torch.zeros(2, 5, 4, 8), torch.zeros(2, 6, 2, 8)
    for call in (lambda: mrf.MrfAttention(q, k, k, 0.5),                                                  # not on the GPU
                 lambda: mrf.MrfAttention(q[0], k, k, 0.5), lambda: mrf.MrfAttention(q, k, k[:, :5], 0.5), lambda: mrf.MrfAttention(q, k.half(), k, 0.5),
                 lambda: mrf.mrf_head_rotation_forward(q, q, None, None, 1e-6, None, q, q), lambda: mrf.mrf_head_rotation_forward(q, k, None, None, 1e-6, None, q, k),
                 lambda: mrf.mrf_gated_scan_forward(q[0], q[0], None, None, q[0], None, None, None), lambda: mrf.mrf_gated_scan_forward(q, q, None, None, q, None, None, None),
                 lambda: mrf.mrf_gated_scan_forward(q[0], q[1].half(), None, None, q[0], None, None, None)):
        with pytest.raises(ValueError):
            call()


def test_attention_backward_workspace_is_for_the_gradients_that_are_asked_for():
    lib = mrf.load_library()
    size = lambda backward, **given: lib.mrf_attention_workspace_bytes(ctypes.byref(_attention(**given)), backward)  # noqa: E731
    table = dict(table=FAKE, bucket_of=FAKE, n_offsets=9, n_buckets=4)
    long = dict(B=1, Hq=32, Hk=32, Q=32768, K=32768)
    # without the table's gradient: as without a table
    assert size(2, **table, **long) == size(1, **long) < 1 << 23
    keeps = size(2, **table)
    assert size(1, **table) > keeps > 0
    back = lambda gt, n: lib.mrf_attention_backward(ctypes.byref(_attention(**table)), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, gt, FAKE, n, None)  # noqa: E731
    assert back(None, keeps - 1) == -6 and back(FAKE, size(1, **table) - 1) == -6 and back(FAKE, keeps) == -6
    # a band: for each 32 keys the queries that see 128 of them, not all there are
    bands = [size(1, **table, B=1, Hq=32, Hk=32, Q=n, K=n, first_offset=-96, last_offset=0) - size(2, B=1, Hq=32, Hk=32, Q=n, K=n) for n in (8192, 32768)]
    assert bands[1] < 4.1 * bands[0] and bands[1] < 32 * 1024 * (96 + 128 + 3 * 64) * 4 + (1 << 20)
    for first, last in ((-(1 << 63), (1 << 63) - 1), (-(1 << 41), 1 << 41), (-40000, 40000), (-(1 << 63), 0)):
        assert size(1, **table, **long, first_offset=first, last_offset=last) == size(1, **table, **long)
    assert size(1, **table, **long, first_offset=5, last_offset=-500) < size(1, **table, **long, first_offset=0, last_offset=0)
    # a large table: as many parts of it as there are offsets for
    many = {**table, "n_buckets": 65536}
    assert size(1, **many) - size(2, **many) < 4 * 65536 * 4 * 8


def test_attention_refuses_more_workgroups_than_a_grid_holds():
    """Workgroups of 512 threads are 2^23 - 1 at most."""
    lib = mrf.load_library()

    def forward(**given):
        return lib.mrf_attention_forward(ctypes.byref(_attention(**given)), FAKE, None, FAKE, 1 << 40, None)

    for bad in (dict(B=1 << 15, Hq=256, Hk=256, Q=100), dict(B=1 << 15, Hq=256, Hk=256, Q=33), dict(B=1 << 15, Hq=256, Hk=128, Q=65), dict(B=1 << 15, Hq=128, Hk=128, Q=257)):
        for t in (1, 2):
            for D in (65, 128):
                assert forward(**bad, type=t, D=D) == -2, bad
                assert lib.mrf_attention_workspace_bytes(ctypes.byref(_attention(**bad, type=t, D=D)), 1) == 0
        # narrower workgroups, of 32 bits and of shorter heads, still fit
        assert lib.mrf_attention_workspace_bytes(ctypes.byref(_attention(**bad, type=0, D=128)), 1) > 0
        assert lib.mrf_attention_workspace_bytes(ctypes.byref(_attention(**bad, type=1, D=64)), 1) > 0
    for good in (dict(B=1 << 15, Hq=255, Hk=255, Q=256), dict(B=1 << 15, Hq=256, Hk=256, Q=32), dict(B=1 << 15, Hq=256, Hk=128, Q=64)):
        assert lib.mrf_attention_workspace_bytes(ctypes.byref(_attention(**good, type=1, D=128, K=1)), 1) > 0


def test_gated_scan_keeps_no_states_where_no_gradient_is_recorded(monkeypatch):
    import torch
    from paper_1910_10892_amd import autograd
    given = []
    monkeypatch.setattr(autograd._m, "mrf_gated_scan_forward", lambda x, z, initial, lengths, y, final, states, *rest: given.append(states))
    x, z = torch.zeros(2, 40, 4, requires_grad=True), torch.zeros(2, 40, 4, requires_grad=True)
    with torch.no_grad():
        autograd.gated_scan(x, z)
    autograd.gated_scan(x.detach(), z.detach())
    autograd.gated_scan(x, z.detach())
    assert given[:2] == [None, None] and given[2].shape == (2, mrf.mrf_gated_scan_states(40), 4)


@pytest.fixture
def bound(monkeypatch):
    """The bindings with tensors of the CPU in place of the GPU's, and calls of the library that work on data noted down instead of made."""
    real, calls = mrf.load_library(), []

    class Library:
        def __getattr__(self, name):
            if name.endswith(("_bytes", "_states", "_strerror")):
                return getattr(real, name)
            return lambda *args: calls.append(name) or 0

    monkeypatch.setattr(binding, "_lib", Library())
    for name in ("_device_of", "_device_now", "_stream_at"):
        monkeypatch.setattr(binding, name, lambda *args: -1)      # (where a tensor of the CPU says that it is)
    return calls


def _refuses(calls, call, good, wrong):
    """The call with its good arguments is made; with one of them wrong at a time it is refused for that one."""
    call(**good)
    assert len(calls) == 1
    for name, value, match in wrong:
        with pytest.raises(ValueError, match=match):
            call(**{**good, name: value})
        assert len(calls) == 1, (name, match)


def _wrong(name, t, more=()):
    """Another shape, another type, other strides of a dense tensor."""
    import torch
    other = torch.int32 if t.dtype == torch.float32 else torch.float32
    yield name, t.new_zeros((*t.shape[:-1], t.shape[-1] + 1)), "%s has shape" % name
    yield name, t.to(other), "%s must be torch" % name
    if t.dim() > 1:
        yield name, t.transpose(0, 1).contiguous().transpose(0, 1), "%s must be contiguous" % name
    yield from more


def test_attention_bindings_refuse_one_wrong_tensor(bound):
    import torch
    q, k, v = torch.zeros(2, 5, 4, 8), torch.zeros(2, 6, 2, 8), torch.zeros(2, 6, 2, 8)
    int32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="tensors must be float32"):
        mrf.MrfAttention(q.double(), k.double(), v.double(), 0.5)
    good = dict(q=q, k=k, v=v, table=torch.zeros(4, 3), bucket_of=int32(11), query_offsets=int32(2), q_lengths=int32(2), k_lengths=int32(2),
                out=torch.zeros(2, 5, 4, 8), lse=torch.zeros(2, 4, 5), scale=0.5)

    def forward(out, lse, scale, q, k, v, **more):
        att = mrf.MrfAttention(q, k, v, scale, **more)
        mrf.mrf_attention_forward(att, out, lse, None)

    wide = lambda t: torch.zeros(*t.shape[:-1], 2 * t.shape[-1])[..., ::2]  # noqa: E731
    wrong = [("q", q[0], "must be"), ("k", k[0], "must be"), ("v", v[0], "v has shape"), ("k", k[:1], "k has shape"), ("k", k[..., :7], "k has shape"), ("v", v[:, :5], "v has shape"),
             ("v", v[:, :, :1], "v has shape"), ("q", q.double(), "must be torch.float64"), ("k", k.half(), "k must be torch"), ("v", v.bfloat16(), "v must be torch"),
             ("q", wide(q), "last index of q"), ("k", wide(k), "last index of k"), ("v", wide(v), "last index of v"), ("bucket_of", None, "bucket_of"),
             ("bucket_of", torch.zeros(11, dtype=torch.int64), "bucket_of must be torch"), ("bucket_of", int32(22)[::2], "bucket_of must be contiguous"),
             ("table", torch.zeros(3, 3), "table has shape"), ("table", torch.zeros(3, 4).t(), "table must be contiguous"),
             ("table", torch.zeros(4, 3).half(), "table must be torch"),
             *_wrong("out", good["out"]), *_wrong("lse", good["lse"])]
    for name in ("query_offsets", "q_lengths", "k_lengths"):
        wrong += [(name, int32(3), "%s has shape" % name), (name, torch.zeros(2, dtype=torch.int64), "%s must be torch" % name), (name, int32(4)[::2], "%s must be contiguous" % name)]
    _refuses(bound, forward, good, wrong)


def test_attention_backward_bindings_refuse_one_wrong_tensor(bound):
    import torch
    q, k = torch.zeros(2, 5, 4, 8), torch.zeros(2, 6, 2, 8)
    att = mrf.MrfAttention(q, k, k, 0.5, table=torch.zeros(4, 3), bucket_of=torch.zeros(11, dtype=torch.int32))
    new = torch.zeros_like
    good = dict(grad_out=new(q), out=new(q), lse=torch.zeros(2, 4, 5), grad_q=new(q), grad_k=new(k), grad_v=new(k), grad_table=torch.zeros(4, 3), workspace=torch.zeros(64, dtype=torch.uint8))
    wrong = [w for name, t in good.items() if name != "workspace" for w in _wrong(name, t)]
    wrong.append(("workspace", torch.zeros(4, 8)[:, ::2], "workspace must be contiguous"))
    _refuses(bound, lambda **a: mrf.mrf_attention_backward(att, **a), good, wrong)
    with pytest.raises(ValueError, match="without a table"):
        mrf.mrf_attention_backward(mrf.MrfAttention(q, k, k, 0.5), **good)
    assert len(bound) == 1


def test_head_rotation_bindings_refuse_one_wrong_tensor(bound):
    import torch
    q, k = torch.zeros(2, 5, 4, 8), torch.zeros(2, 5, 2, 8)
    new = torch.zeros_like
    inputs = dict(q=q, k=k, gamma_q=torch.ones(8), gamma_k=torch.ones(8), eps=1e-6, inv_freq=torch.ones(4), positions=torch.zeros(2, 5, 2, dtype=torch.int32))
    wide = torch.zeros(2, 5, 4, 16)[..., ::2]
    wrong = [("q", q[0], "must be"), ("k", k[0], "must be"), ("k", k[:, :4], "k has shape"), ("k", k[..., :7], "k has shape"), ("q", q.double(), "tensors must be float32"),
             ("k", k.half(), "k must be torch"), ("q", wide, "last index of q"), ("k", wide[:, :, :2], "last index of k"), ("inv_freq", torch.ones(4).half(), "inv_freq must be torch"),
             ("inv_freq", torch.ones(8)[::2], "inv_freq must be contiguous"), ("positions", torch.zeros(2, 4, dtype=torch.int32), "positions has shape"),
             ("positions", torch.zeros(2, 5), "positions must be torch"), ("positions", torch.zeros(2, 5, 4, dtype=torch.int32)[..., ::2], "positions must be contiguous")]
    for name in ("gamma_q", "gamma_k"):
        wrong += [*_wrong(name, torch.ones(8)), (name, torch.ones(16)[::2], "%s must be contiguous" % name)]
    forward = {**inputs, "out_q": new(q), "out_k": new(k)}
    _refuses(bound, mrf.mrf_head_rotation_forward, forward, wrong + [*_wrong("out_q", q), *_wrong("out_k", k)])
    bound.clear()
    grads = dict(grad_out_q=new(q), grad_out_k=new(k), grad_q=new(q), grad_k=new(k), grad_gamma_q=torch.ones(8), grad_gamma_k=torch.ones(8))
    _refuses(bound, mrf.mrf_head_rotation_backward, {**inputs, **grads, "workspace": torch.zeros(64, dtype=torch.uint8)}, wrong + [w for n, t in grads.items() for w in _wrong(n, t)])


def test_gated_scan_bindings_refuse_one_wrong_tensor(bound):
    import torch
    x = torch.zeros(2, 40, 4)
    new = torch.zeros_like
    ends, states, lengths = torch.zeros(2, 4), torch.zeros(2, mrf.mrf_gated_scan_states(40), 4), torch.zeros(2, dtype=torch.int32)
    wide = torch.zeros(2, 40, 8)[..., ::2]
    inputs = dict(x=x, z=new(x), lengths=lengths, states=states, workspace=None)
    wrong = [("x", x[0], "must be"), ("z", x[0], "z has shape"), ("z", x[:, :39], "z has shape"), ("z", x.half(), "z must be torch"), ("x", x.double(), "tensors must be float32"),
             ("x", wide, "last index of x"), ("z", wide, "last index of z"), ("lengths", lengths.long(), "lengths must be torch"), ("lengths", torch.zeros(3, dtype=torch.int32), "lengths has shape"),
             ("lengths", torch.zeros(4, dtype=torch.int32)[::2], "lengths must be contiguous"), *_wrong("states", states)]
    more = lambda given: wrong + [w for n, t in given.items() for w in _wrong(n, t)]  # noqa: E731
    forward = dict(initial=ends, y=new(x), final=new(ends))
    _refuses(bound, mrf.mrf_gated_scan_forward, {**inputs, **forward}, more(forward))
    bound.clear()
    grads = dict(grad_y=new(x), grad_final=new(ends), grad_x=new(x), grad_z=new(x), grad_initial=new(ends))
    _refuses(bound, mrf.mrf_gated_scan_backward, {**inputs, **grads}, more(grads))


def test_numbers_that_a_description_cannot_hold_are_refused_as_such(bound):
    import torch
    q, k, table, bucket_of = torch.zeros(2, 5, 4, 8), torch.zeros(2, 6, 2, 8), torch.zeros(4, 3), torch.zeros(11, dtype=torch.int32)
    attention = dict(q=q, k=k, v=k, scale=0.5, table=table, bucket_of=bucket_of)
    for wrong in (dict(first_offset=1 << 63), dict(last_offset=-(1 << 64)), dict(query_offset=1 << 70), dict(map_offset=1 << 63),
                  dict(table=torch.zeros(3)), dict(table=torch.zeros(()))):
        with pytest.raises(ValueError):
            mrf.MrfAttention(**{**attention, **wrong})
    mrf.MrfAttention(**attention, first_offset=-(1 << 63), last_offset=(1 << 63) - 1)
    for wrong in (dict(position_offset=1 << 63), dict(position_offset=-(1 << 64))):
        with pytest.raises(ValueError):
            mrf.mrf_head_rotation_forward(q, q, None, None, **{**dict(eps=1e-6, inv_freq=None, out_q=q, out_k=q), **wrong})
    assert bound == []


def test_strides_of_tensors_without_elements_do_not_matter(bound):
    import torch
    q, x = torch.zeros(2, 5, 4, 8), torch.zeros(2, 40, 4)
    none = torch.empty_strided((2, 5, 0, 8), (0, 0, 0, 3))
    mrf.mrf_head_rotation_forward(q, none, None, None, 1e-6, None, q, none)
    no_keys = torch.empty_strided((2, 0, 2, 8), (0, 0, 0, 3))
    mrf.mrf_attention_forward(mrf.MrfAttention(q, no_keys, no_keys, 0.5), q, None, None)
    no_steps = torch.empty_strided((2, 0, 4), (0, 0, 3))
    mrf.mrf_gated_scan_forward(no_steps, no_steps, None, None, x[:, :0].contiguous(), None, None, None)
    assert len(bound) == 3
