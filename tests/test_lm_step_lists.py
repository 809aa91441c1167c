"""Lists of gradients that were laid out once: tensors that are not any more what they were are refused before anything is launched, so no GPU is needed (the tensors are the CPU's)."""
import ctypes as C

import pytest
import torch

import paper_2009_05766_amd as nm
from paper_2009_05766_amd import lm_step_ops


def laid(*tensors):
    entries = (nm.netmax_gradient * len(tensors))()
    for e, t in zip(entries, tensors):
        e.g, e.out, e.rows, e.cols, e.ldg, e.ldo, e.dtype = t.data_ptr(), t.data_ptr(), 1, t.numel(), t.numel(), t.numel(), lm_step_ops._DTYPES[t.dtype]
    return entries, lm_step_ops._laid_out(tensors + tensors)


def call(tensors, entries, layout):
    """A call of netmax_grad_norm as Gradients makes it."""
    (lm_step_ops._calls or lm_step_ops._load_calls()).clip(tensors, tensors, layout, C.addressof(entries), 1, False, None)


def transposed(t):
    t.t_()


CHANGES = [("reshaped", lambda t: t.resize_(15, 60), "changed"), ("flattened", lambda t: t.resize_(900), "changed"), ("emptied", lambda t: t.resize_(0, 30), "moved"),
           ("transposed", transposed, "changed"), ("strided", lambda t: t.as_strided_((30, 10), (30, 1)), "changed"), ("moved", lambda t: setattr(t, "data", torch.zeros(30, 30)), "moved"),
           ("offset", lambda t: t.as_strided_((30, 29), (30, 1), 1), "moved"), ("dimension", lambda t: t.unsqueeze_(0), "changed")]


@pytest.mark.parametrize("k", range(len(CHANGES)), ids=[c[0] for c in CHANGES])
def test_changed_tensors_are_refused(k):
    _, change, text = CHANGES[k]
    tensors = (torch.zeros(7), torch.zeros(30, 30), torch.zeros(5, 3, dtype=torch.bfloat16))
    entries, layout = laid(*tensors)
    change(tensors[1])
    with pytest.raises(nm.NetmaxError, match=text) as e:
        call(tensors, entries, layout)
    assert e.value.code == nm.NETMAX_EINVAL


def test_another_type_is_refused():
    tensors = (torch.zeros(6, dtype=torch.bfloat16),)
    entries, layout = laid(*tensors)
    other = tensors[0].view(torch.int16)                            # the same memory
    with pytest.raises(nm.NetmaxError, match="type"):
        call((other,), entries, layout)


def test_a_list_of_other_tensors_is_refused():
    tensors = (torch.zeros(7), torch.zeros(30, 30))
    entries, layout = laid(*tensors)
    for given, bytes_ in (((tensors[0],), layout), (tensors, layout[:-8]), (tensors, layout + bytes(8)), (tensors, layout[:40]), (tensors, b""), ((tensors[1], tensors[0]), layout)):
        with pytest.raises(nm.NetmaxError) as e:
            call(given, entries, bytes_)
        assert e.value.code == nm.NETMAX_EINVAL
