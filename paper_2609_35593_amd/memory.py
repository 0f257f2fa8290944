"""Memory of the calls that the binding makes on a stream, from torch's caching allocator."""
from __future__ import annotations

import torch

# A device's current stream as an address, without a Stream object around it, where torch offers that.
raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _side(stream, device):
    """The caller's stream, where it is not torch's current one."""
    if stream is None:
        return None
    address = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    if address == raw_stream(device.index):
        return None
    return stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(address, device=device)


def empty(shape, dtype, device, stream, strides=None, output=True):
    """An output or workspace. For a stream that is not torch's current one it is that stream's memory: a block of the
    current one's may still be in use by work queued there, which the other does not wait for. An output is marked as
    in use on the current stream as well, where the caller may go on with it."""
    make = lambda: (torch.empty(shape, dtype=dtype, device=device) if strides is None
                    else torch.empty_strided(shape, strides, dtype=dtype, device=device))
    side = _side(stream, device)
    if side is None:
        return make()
    with torch.cuda.stream(side):
        t = make()
    if output:
        t.record_stream(torch.cuda.current_stream(device))
    return t
