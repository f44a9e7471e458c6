"""Norm and rotation in front of the head-sharded call run where the exchanges and attention behind them run."""
import pytest

from paper_2609_37001_b200 import ulysses as U
from test_ulysses_gloo import GRID, PARAMS, SCALE, TILE, _full_inputs, _oracle_attn


def test_a_stream_of_its_own_is_refused():
    """On another stream the exchanges and attention, on the current one, would read q and k before they are written."""
    q, k, v = _full_inputs()
    called = []

    def norm_rope_fn(q, k, grid, first_token=0, stream=None):
        called.append(stream)
        return q, k

    def call(options):
        return U.psa_attn_fwd_ulysses(q, k, v, PARAMS, GRID, TILE, SCALE, attn_fn=_oracle_attn, norm_rope=options, norm_rope_fn=norm_rope_fn)

    with pytest.raises(ValueError):
        call(dict(stream=object()))
    assert called == []
    call(dict(stream=None))
    assert called == [None]
