"""The oracle's decode rates where the first forward is slow (no GPU is needed)."""

import time

import bench
import oracle
import sd_synth as S


def test_a_slow_first_forward_does_not_make_a_rate_negative(monkeypatch):
    """Threads start and weights are touched in the first forward, which then takes longer than a tiny
    model's prefill and decode together; it must not be what is taken off them."""
    forward, calls = oracle.Model.forward, []

    def slow_at_first(self, *args, **kwargs):
        calls.append(0)
        if len(calls) == 1:
            time.sleep(1.0)
        return forward(self, *args, **kwargs)

    monkeypatch.setattr(oracle.Model, "forward", slow_at_first)
    wl, cfg = S.WORKLOADS["tiny"], S.MODELS["tiny"]
    r = bench.oracle_decode_rates(cfg, S.make_weights(cfg, 0), S.prompt(cfg, wl.prompt_len), wl, S.skip_mask(cfg, wl.mask))
    assert r["sd_tokens_per_s"] > 0 and r["ar_tokens_per_s"] > 0 and r["prefill_s"] < 1.0
