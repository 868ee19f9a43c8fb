"""What the binding of the paged cache's operators refuses before it hands addresses to the library.  The tensors here are host
tensors that say they are on a GPU: a call that is not refused ends at the missing GPU, not in a launch."""
import pytest
import torch

import paper_2507_05228_amd as cas


class OnGpu(torch.Tensor):
    """A host tensor that claims to be on GPU `device`."""
    device_id = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.device_id


def gpu(t, device=0):
    t = t.as_subclass(OnGpu)
    t.device_id = device
    return t


def i32(*shape):
    return gpu(torch.zeros(shape, dtype=torch.int32))


def heads(rows, n, d=64):
    return gpu(torch.zeros(rows, n, d, dtype=torch.bfloat16))


def broadcast(rows, n, d=64):
    return gpu(torch.zeros(1, n, d, dtype=torch.bfloat16).expand(rows, n, d))


def overlapping(rows, n, d=64):
    return gpu(torch.zeros(rows * n * d, dtype=torch.bfloat16).as_strided((rows, n, d), (d, d, 1)))


def pool(device=0):
    return cas.make_paged_cache(heads(8, 2).new_zeros(1, 4, 2, 16, 64), heads(8, 2).new_zeros(1, 4, 2, 16, 64), i32(2, 1, 3), i32(2, 1), i32(4))


def refused(status, call, *args, **kw):
    with pytest.raises(cas.CascadeError) as e:
        call(*args, **kw)
    assert e.value.status == status


@pytest.mark.parametrize("odd", [broadcast, overlapping])
def test_rows_that_share_memory(odd):
    """A row stride of 0 is the library's word for dense rows: a broadcast would be read, or written, far beyond its one row."""
    rope, pos, cache = cas.make_rope_desc(64, 1e4), i32(3), pool()
    refused(cas.ESHAPE, cas.cascade_rope, rope, odd(3, 4), pos)
    refused(cas.ESHAPE, cas.cascade_rope, rope, odd(3, 4), pos, heads(3, 4))
    refused(cas.ESHAPE, cas.cascade_rope, rope, heads(3, 4), pos, odd(3, 4))
    slots, k, q = i32(3), heads(3, 2), heads(3, 4)
    refused(cas.ESHAPE, cas.cascade_paged_append, cache, 0, slots, odd(3, 2), odd(3, 2))
    refused(cas.ESHAPE, cas.cascade_paged_append, cache, 0, slots, k, k, positions=pos, rope=rope, q=odd(3, 4))
    refused(cas.ESHAPE, cas.cascade_paged_append, cache, 0, slots, k, k, positions=pos, rope=rope, q=q, q_out=odd(3, 4))
    q_start = i32(3)
    refused(cas.ESHAPE, cas.cascade_paged_attn, cache, 0, odd(3, 4), q, q_start, 0.1)
    refused(cas.ESHAPE, cas.cascade_paged_attn, cache, 0, q, odd(3, 4), q_start, 0.1)
