"""GPU: dispatch and combine under autograd when a program reuses buffers."""
import pytest

pytestmark = pytest.mark.gpu


def _inputs(T=40, k=2, H=72, E=4):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(0)
    ids = torch.randint(0, E, (T, k), dtype=torch.int32, device="cuda", generator=gen)
    gates = torch.rand(T, k, device="cuda", generator=gen)
    return ids, gates, torch.randn(T, H, device="cuda", generator=gen)


def _changes_of_saved_tensors():
    """name -> what a program does between a forward pass and its backward pass with
    y, the gates and the routing that the forward pass saved, through each call that
    writes to a tensor that it is given."""
    from paper_2609_07536_amd import experts as X
    return {
        "sort": lambda ids, x, y, r: X.sort_by_expert(ids.flip(0), r.gate_w.view(ids.shape), 4, out=r),
        "dispatch": lambda ids, x, y, r: X.dispatch_rows(x, r.slot_rows, y.shape[0], out=y),
        "dispatch_grad": lambda ids, x, y, r: X.dispatch_rows_grad(y.clone(), r.slot_rows, out=y[:len(x)]),
        "combine": lambda ids, x, y, r: X.combine_rows(y.clone(), r.slot_rows, r.gate_w.view(ids.shape), out=y[:len(x)]),
        "combine_grad": lambda ids, x, y, r: X.combine_rows_grad(
            x, y.clone(), r.slot_rows, r.gate_w.view(ids.shape), out=(y, x.new_empty(ids.shape))),
        "dequantize": lambda ids, x, y, r: X.mx4_dequantize(X.mx4_quantize(y), out=y),
    }


@pytest.mark.parametrize("name", ["sort", "dispatch", "dispatch_grad", "combine", "combine_grad", "dequantize"])
def test_a_saved_tensor_that_a_call_wrote_to_is_refused(gpu_lib, name):
    """As after torch's own in-place operations: an error, not another gradient."""
    import torch

    from paper_2609_07536_amd import autograd as A
    from paper_2609_07536_amd import experts as X
    ids, gates, x = _inputs()
    r = X.sort_by_expert(ids, gates, 4)
    y = X.dispatch_rows(x, r.slot_rows, ids.numel())
    g = gates.clone().requires_grad_()
    out = A.combine(y, r, g)
    _changes_of_saved_tensors()[name](ids, x, y, r)
    with pytest.raises(RuntimeError, match="inplace"):
        out.sum().backward()
    if name == "sort":
        w = x.clone().requires_grad_()
        rows = A.dispatch(w, r)
        _changes_of_saved_tensors()[name](ids, x, y, r)
        with pytest.raises(RuntimeError, match="inplace"):
            rows.sum().backward()


def test_every_given_output_counts_as_changed(gpu_lib):
    """... and nothing that a call only reads."""
    import torch

    from paper_2609_07536_amd import experts as X
    ids, gates, x = _inputs()
    T, k, H, E, I = *ids.shape, x.shape[1], 4, 32
    r = X.sort_by_expert(ids, gates, E)
    y = X.dispatch_rows(x, r.slot_rows, T * k)
    a = X.mx4_quantize(x)
    w = X.mx4_quantize_weights(torch.randn(E, H, 2 * I, device="cuda"))
    w2 = X.mx4_quantize_weights(torch.randn(E, I, H, device="cuda"))
    wide, h = torch.randn(E, H, 2 * I, device="cuda"), x.bfloat16()
    inputs = [ids, gates, x, y, wide, h, *r, *a[:2], *w[:2], *w2[:2]]
    calls = [
        (lambda out: X.sort_by_expert(ids, gates, E, out=out), [torch.empty_like(t) for t in r]),
        (lambda out: X.dispatch_rows(x, r.slot_rows, T * k, out=out), torch.empty_like(y)),
        (lambda out: X.dispatch_rows_grad(y, r.slot_rows, out=out), torch.empty_like(x)),
        (lambda out: X.combine_rows(y, r.slot_rows, gates, out=out), torch.empty_like(x)),
        (lambda out: X.combine_rows_grad(x, y, r.slot_rows, gates, out=out), [torch.empty_like(y), torch.empty_like(gates)]),
        (lambda out: X.mx4_quantize(x, out=X.MX4(*out, H)), [torch.empty_like(t) for t in a[:2]]),
        (lambda out: X.mx4_quantize_weights(wide, out=X.MX4(*out, H)), [torch.empty_like(t) for t in w[:2]]),
        (lambda out: X.mx4_dequantize(a, out=out), torch.empty_like(x)),
        (lambda out: X.mx4_product(a, w, r.expert_offsets, T * k, row_ids=r.token_ids, swiglu=True, out=out),
         torch.empty(T * k, I, dtype=torch.bfloat16, device="cuda")),
        (lambda out: X.layer_forward_mx4(h, w, w2, r, gates, out=out), torch.empty_like(x)),
    ]
    before = [t._version for t in inputs]
    for call, out in calls:
        outs = [out] if isinstance(out, torch.Tensor) else out
        was = [t._version for t in outs]
        call(out)
        assert all(t._version > v for t, v in zip(outs, was)), call
    assert [t._version for t in inputs] == before


def test_rows_of_another_number_and_types_without_a_gradient_are_refused(gpu_lib):
    """A y that is short of rows, and a gradient that no kernel has, when the forward pass
    is asked for them."""
    import torch

    from paper_2609_07536_amd import autograd as A
    from paper_2609_07536_amd import experts as X
    ids, gates, x = _inputs()
    r = X.sort_by_expert(ids, gates, 4)
    y = A.dispatch(x, r)
    for bad in (y[:-1], y[:0], torch.cat((y, y[:1]))):
        with pytest.raises(TypeError):
            A.combine(bad, r, gates)
    for dtype in (torch.float16, torch.float64):
        with pytest.raises(TypeError):
            A.dispatch(x.to(dtype).requires_grad_(), r)
        rows = A.dispatch(x.to(dtype), r)    # moved as they are
        assert rows.dtype == dtype and torch.equal(rows[r.slot_rows[3, 1]], x[3].to(dtype))
        with torch.no_grad():
            assert torch.equal(A.dispatch(x.to(dtype).requires_grad_(), r), rows)


def test_bad_slots_are_flagged_in_both_directions(gpu_lib):
    import torch

    from paper_2609_07536_amd import autograd as A
    from paper_2609_07536_amd import binding as B
    from paper_2609_07536_amd import experts as X
    ids, gates, x = _inputs()
    good = X.sort_by_expert(ids, gates, 4)
    slots = good.slot_rows.clone()
    slots[2, 1] = slots.numel() + 3
    bad, ws = good._replace(slot_rows=slots), B.Workspace(512)
    for routing, code in ((good, 0), (bad, B.MOE_ERR_BAD_ROUTING)):
        leaf, g = x.clone().requires_grad_(), gates.clone().requires_grad_()
        rows = A.dispatch(leaf, routing, workspace=ws)
        assert ws.status(clear=True) == code
        rows.sum().backward()
        assert ws.status(clear=True) == code
        y = rows.detach().requires_grad_()
        out = A.combine(y, routing, g, workspace=ws)
        assert ws.status(clear=True) == code
        out.sum().backward()
        assert ws.status(clear=True) == code
