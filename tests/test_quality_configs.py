"""Which configurations the quality sweep runs (on the host: the linears
themselves are replaced)."""
import dataclasses

import pytest
import torch

from paper_2406_18832_amd import quality, synth

ALL = [c[0] for c in quality.CONFIGS]
MX4 = [c[0] for c in quality.MX4_CONFIGS]


@pytest.fixture
def workload(monkeypatch):
    """A workload of one linear whose 48 channels are no whole blocks of 32, and one
    of 64; the int8 linears replaced by the float one."""
    wl = dataclasses.replace(synth.WORKLOADS["opt125m_w8a8"], name="odd",
                             layers=(synth.Layer("odd", 48, 8), synth.Layer("even", 64, 8)))
    monkeypatch.setitem(synth.WORKLOADS, "odd", wl)

    def inputs(wl, li, rows, *rest):
        g = torch.Generator().manual_seed(li)
        lay = wl.layers[li]
        return (torch.randn(rows, lay.K, generator=g).half(), torch.randn(lay.N, lay.K, generator=g).half(),
                torch.randn(lay.N, generator=g).half(), torch.zeros(2 * lay.K))
    monkeypatch.setattr(quality, "layer_inputs", inputs)
    run = quality.run_config

    def config(X, W, b, minmax, a_bits, w_bits, path):
        if path.startswith("mx4") and X.shape[1] % 32:
            return run(X, W, b, minmax, a_bits, w_bits, "mx4-plain")  # raises
        return (X.double() @ W.double().t() + b.double()).half()
    monkeypatch.setattr(quality, "run_config", config)
    return "odd"


def test_layers_without_whole_blocks_run_without_mx4(workload):
    recs = quality.sweep(workloads=(workload,), rows=5)
    by = {name: [r["config"] for r in recs if r["layer"] == name] for name in ("odd", "even")}
    assert by == {"odd": ALL, "even": ALL + MX4}


def test_a_configuration_asked_for_is_not_left_out(workload):
    with pytest.raises(ValueError, match="multiple of 32"):
        quality.sweep(workloads=(workload,), rows=5, configs=quality.MX4_CONFIGS)
    recs = quality.sweep(workloads=(workload,), rows=5, configs=quality.CONFIGS[:2])
    assert [r["config"] for r in recs] == 2 * ALL[:2]
