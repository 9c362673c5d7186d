"""What the binding of the sequence memory says of arguments that are no tensors, or of too few dimensions: an HtsError that names them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_it_names_what_is_missing():
    import paper_2012_09849_amd as hts
    T, N, D, S = 3, 2, 8, 4
    new = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    x, pair, A, w = new(T, N, D), new(T, N, S), new(D, S), new(D, 4)
    states = new(hts.selective_scan_states(T, N, D, S))
    ctx = hts.SeqContext(max(hts.short_conv_workspace(T, N, D, 4), hts.selective_scan_workspace(T, N, D, S)))
    for bad in (None, 3, new(D)):
        with pytest.raises(hts.HtsError, match="w:"):
            ctx.hts_short_conv(x, bad, x.clone())
        with pytest.raises(hts.HtsError, match="w:"):
            ctx.hts_short_conv_backward(x, bad, x, x.clone(), w.clone())
        with pytest.raises(hts.HtsError, match="A:"):
            ctx.hts_selective_scan(x, x, bad, pair, pair, x.clone())
        with pytest.raises(hts.HtsError, match="B:"):
            ctx.hts_selective_scan(x, x, A, bad, pair, x.clone())
        with pytest.raises(hts.HtsError, match="w:"):
            ctx.hts_linear(x[0], bad, x[0].clone())
    for bad in ([1.0], states[:-1]):
        with pytest.raises(hts.HtsError, match="states:"):
            ctx.hts_selective_scan(x, x, A, pair, pair, x.clone(), states=bad)
    for bad in (None, states[:-1]):
        with pytest.raises(hts.HtsError, match="states:"):
            ctx.hts_selective_scan_backward(x, x, A, pair, pair, x, bad, x.clone(), x.clone(), pair.clone(), pair.clone(), A.clone())
    ctx.close()
