"""Gated dense layers in the host-side partitioning: split, listed and counted like
dense ones, with two projections.  No GPU."""
import pytest

from paper_2112_15317_amd import configs
from paper_2112_15317_amd import partition as P


def _net(gate="silu"):
    return P.vgg_net(configs.PAPER_VARIANT_CONV, 3, 32, configs.PAPER_VARIANT_FC, gate=gate)


def test_gated_layers_are_split_like_dense_ones():
    assert P.fc_plan(P.partition(_net(), 2)) == [
        ("modulo", 4096), ("gated", 4096, 512, 1024, "silu"), ("shard", 512, 1024),
        ("gated", 1024, 512, 1024, "silu"), ("shard", 512, 1024), ("linear", 1024, 5, 10, False),
        ("shard", 5, 10), ("loss", 10)]
    assert P.fc_shards(P.partition(_net("gelu"), 2)) == [(4096, 512, 1024), (1024, 512, 1024), (1024, 5, 10)]


def test_counts_two_projections():
    layers = [P.gated(8, 6)]
    assert P.parameters(layers) == 2 * (8 * 6 + 6)
    assert P.ccr(P.gated(8, 6)) == 2 * P.ccr(P.linear(8, 6))


def test_refusals():
    with pytest.raises(ValueError):
        P.gated(8, 6, "tanh")
    net = P.seq(P.gated(64, 32), P.Layer(P.RELU), P.linear(32, 8), P.Layer(P.LOG_SOFTMAX))
    with pytest.raises(ValueError):
        P.fc_plan(P.partition(net, 2))
    with pytest.raises(ValueError):
        P.partition(P.seq(P.gated(64, 33), P.Layer(P.LOG_SOFTMAX)), 2)
