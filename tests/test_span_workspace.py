"""The workspace of attn_span_bwd on very long sequences (host only)."""
import pytest

import paper_2609_03151_amd as basp


@pytest.mark.parametrize("n_q,n_k,d", [(1, 1, 128), (2, 1, 64), (4, 4, 64), (3, 1, 80), (1, 1, 96)])
def test_grows_with_the_length(n_q, n_k, d):
    """At most 16 partial sums of dK and dV, as the causal backward keeps, whatever the length; beside
    them four numbers a row and head (the causal backward keeps two), four a row, and per 32 rows a
    hull and per unit a flag."""
    longest = -(-2 ** 31 // (n_q * d * 2)) - 256      # (S + 256) rows of 2^31 bytes are refused
    for S in (4096, 131072, 1 << 20, (1 << 20) + 1, 1500007, 1 << 21, 3 << 20, 1 << 22, longest - 1,
              longest):
        need = basp.attn_span_bwd_workspace_bytes(1, S, n_q, n_k, d)
        if S >= longest:
            assert need == 0
            continue
        if S > longest:
            continue
        rows = S + 64
        assert need <= (2 * 16 * S * n_k * d * 4 + rows * (16 * n_q + 16 + 1) + 16 * n_k * (rows // 128 + 1)
                        * 4 + 2048), S
        if S >= 1 << 20:
            causal = basp.attn_bwd_workspace_bytes(1, S, n_q, n_k, d, 1)
            assert need <= causal + rows * (8 * n_q + 17) + 16 * n_k * (rows // 128 + 1) * 4 + 2048, S
