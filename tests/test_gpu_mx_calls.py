"""Calls of the microscaled 4-bit operators at the edges of what the header allows."""
import numpy as np
import pytest

import mx_plain

pytestmark = pytest.mark.gpu


def _mx():
    from paper_2106_05373_amd import mx
    return mx


def _bcpnn():
    from paper_2106_05373_amd import bcpnn
    return bcpnn


def _gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def test_a_layer_whose_inputs_broke_their_pairs_is_not_copied():
    """Making a copy waits for the stream, so it reports what training saw of the inputs."""
    import torch
    B = _bcpnn()
    cfg = B.default_config(64, 2, 4, 16, 32, complement_pairs=1)
    pixels = torch.rand(32, 64, generator=_gen(1), device="cuda")
    x = torch.stack([pixels, 1 - pixels], 2).reshape(32, 128).contiguous()
    with B.Layer(cfg) as layer:
        layer.train_batch(x)
        _mx().Layer.of(layer).close()
        x[5, 7] += 0.25
        layer.train_batch(x)
        with pytest.raises(B.BcpnnError, match="EINPUT"):
            _mx().Layer.of(layer)
        with pytest.raises(B.BcpnnError, match="ESTATE"):
            _mx().Layer.of(layer)
