"""The calls are handed to the library past torch's dispatcher, so that a trace would hold the results' memory and not what fills it: refused, on the host, before any launch."""
import pytest
import torch
from torch.fx.experimental.proxy_tensor import make_fx

import paper_2508_18224_amd as nsa
from test_call_transforms import NAMES, _calls


@pytest.mark.parametrize("name", NAMES)
def test_tracing_is_refused(name):
    call, x = _calls()[name]
    with pytest.raises(nsa.NsaSelError, match="trace"):
        torch.jit.trace(call, (x,), check_trace=False)
    for pre_dispatch in (False, True):
        with pytest.raises(nsa.NsaSelError, match="trace"):
            make_fx(call, pre_dispatch=pre_dispatch)(x)
