"""The word of a device in which products of 16-bit and of 4-bit operands report a wait that ran out (see ``include/signsgd.h``, status)."""
from __future__ import annotations

import threading
from typing import Tuple

import torch

_status = {}
_making = threading.Lock()


def status_of(device: torch.device) -> Tuple[torch.Tensor, int]:
    """The word of a device, and its address."""
    s = _status.get(device)
    if s is None:
        with _making:                           # one word for all threads: a kernel may hold the address of each that was given out
            s = _status.get(device)
            if s is None:
                if torch.cuda.is_current_stream_capturing():
                    raise RuntimeError("the first such call on a device must come before any stream capture")
                t = torch.zeros(1, dtype=torch.int32, device=device)
                torch.cuda.synchronize(device)  # zero before a product on any stream may use it
                s = _status[device] = (t, t.data_ptr())
    return s


def check(device="cuda") -> None:
    """Waits for the device and raises if a product since the last check had to give up a bounded wait."""
    device = torch.device("cuda", torch.cuda.current_device()) if torch.device(device).index is None else torch.device(device)
    s = status_of(device)[0]
    torch.cuda.synchronize(device)
    if int(s.item()):
        s.zero_()
        raise RuntimeError("a product did not receive its operands in time; its output is not valid")
