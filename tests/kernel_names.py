"""The names of the library's kernels that a call launches."""
import warnings

import torch
from torch.profiler import ProfilerActivity, profile


def launched(call):
    """(what the call returned, the names in the order of their start)"""
    torch.cuda.synchronize()
    with warnings.catch_warnings():
        warnings.simplefilter("ignore")
        with profile(activities=[ProfilerActivity.CUDA]) as p:
            out = call()
            torch.cuda.synchronize()
        names = [e.name for e in sorted(p.events(), key=lambda e: e.time_range.start) if "igc::" in e.name]
    assert names, "the profiler saw no kernel of the library"
    return out, names
