"""Logits of other widths than the vocabulary: rows that are too short are refused, whatever their distance (CPU), and
a model's handle knows its vocabulary (GPU)."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")
tadm = pytest.importorskip("paper_2609_37924_amd")


@pytest.mark.parametrize("R", [1, 3])
def test_rows_that_are_too_short(R):
    m = C.c_void_p()  # a null model: what is not refused before says so
    m.vocab = 64
    full, u, token = torch.zeros(R, 80), torch.zeros(R), torch.zeros(R, dtype=torch.int32)
    for logits in (full[:, 17:], full[:, :63], full[:, 79:], torch.zeros(R, 64)[:, 1:] if R > 1 else full[:, 20:]):
        assert logits.stride(0) >= 64
        with pytest.raises(ValueError, match="vocabulary of 64"):
            tadm.tadm_sample_rows(m, logits, None, u, token)
    for logits in (full[:, :64], full[:, 16:], full, torch.zeros(R, 64)):
        with pytest.raises(tadm.TadmError, match="null model"):
            tadm.tadm_sample_rows(m, logits, None, u, token)


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")
def test_a_model_refuses_them():
    import synth
    m = tadm.tadm_model_create(tadm.make_config(synth.get_config("tiny", vocab=300), max_batch=1, max_seq=64))
    tadm.tadm_set_stream(m, torch.cuda.current_stream().cuda_stream)
    try:
        full, u, token = torch.zeros(4, 364, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
        full[:, 300:] = 9.0  # behind the vocabulary
        full[:, 70] = 5.0
        with pytest.raises(ValueError, match="vocabulary of 300"):
            tadm.tadm_sample_rows(m, full[:, 65:], None, u, token)
        greedy = tadm.row_settings(temperature=torch.zeros(4, device="cuda"))
        for logits in (full, full[:, :300]):
            token.fill_(-7)
            tadm.tadm_sample_rows(m, logits, greedy, u, token, None, None)
            assert token.tolist() == [70] * 4
    finally:
        tadm.tadm_model_destroy(m)
