"""The residual gated block's Python methods refuse tensors of another device than the handle's, before any
entry point is called. Tensors that say where they are stand in for a second GPU's."""
import pytest

torch = pytest.importorskip("torch")

from paper_2407_09486_amd import blocks  # noqa: E402


class _On(torch.Tensor):
    """A tensor whose device has the index `where`."""
    where = 0

    @property
    def is_cuda(self):
        return True

    def get_device(self):
        return self.where


def on(index, *shape, dtype=torch.float32):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(_On)
    t.where = index
    return t


def unopened(kind, **fields):
    op = object.__new__(kind)
    op._device, op.handle = 0, None
    for k, v in fields.items():
        setattr(op, k, v)
    return op


def each_elsewhere(call, names, shapes, match=None):
    """call(**tensors) with one of them on device 1 at a time."""
    for bad in names:
        t = {n: on(1 if n == bad else 0, *shapes[n]) for n in shapes}
        with pytest.raises(ValueError, match=f"{(match or {}).get(bad, bad)}.*cuda:0"):
            call(**t)


def test_gated_block():
    op = unopened(blocks.GatedBlock, dtype=torch.float32, model=4, hidden=6, _saved_floats=lambda rows: 30)
    w = dict(x=(3, 4), wg=(6, 4), wu=(6, 4), wd=(4, 6))
    each_elsewhere(op.forward, [*w, "y", "saved"], {**w, "y": (3, 4), "saved": (30,)})
    each_elsewhere(op.backward, [*w, "dy", "saved"], {**w, "dy": (3, 4), "saved": (30,)})


def test_residual_norm():
    op = unopened(blocks.ResidualNorm, dtype=torch.float32, model=4, group=2)
    t = dict(residual=(3, 4), branch=(3, 4), post=(4,), pre=(4,), post_bias=(4,), pre_bias=(4,), gate=(2, 4))
    each_elsewhere(op.forward, t, t)
    t.update(dres=(3, 4), dout=(3, 4), stats=(3, 4))
    each_elsewhere(op.backward, t, t)


def test_adamw(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    names = ("params", "grads", "copies", "m", "v", "m_scale", "v_scale")
    types = dict(copies=torch.bfloat16, m=torch.int8, v=torch.uint8)
    for bad in names:
        t = {n: [on(1 if n == bad else 0, 1 if "scale" in n else 5, dtype=types.get(n, torch.float32))] for n in names}
        with pytest.raises(ValueError, match=rf"{bad}\[0\].*cuda:0"):
            blocks.AdamW(bits=8, **t)
    op = unopened(blocks.AdamW, _grad_type=torch.float32, _sizes=[5], bits=8)
    with pytest.raises(ValueError, match="grads"):
        op.set_grads([on(1, 5)])
    with pytest.raises(ValueError, match="states"):
        op.states([on(0, 5)], [on(1, 5)])


def test_int8_linear(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    t = dict(codes=(6, 16), scales=(6,), bias=(6,))
    for bad in t:
        v = {n: on(1 if n == bad else 0, *t[n], dtype=torch.int8 if n == "codes" else torch.float32) for n in t}
        with pytest.raises(ValueError, match=f"{bad}.*cuda:0"):
            blocks.Int8Linear(**v)
    op = unopened(blocks.Int8Linear, dtype=torch.float32, columns=16, outputs=6)
    each_elsewhere(op.__call__, ["x", "y"], dict(x=(3, 16), y=(3, 6)))
