"""GPU tests of uniprefill_attention in work-groups of 256 rows: every type and head dimension, keys whole and cut into
pieces, packed and in pages of two sizes (tests/test_host_attention_forms.py checks that the batches are of these forms)."""
import pytest

from attention_form_cases import FORMS, TYPES
from oracle import attention_oracle as ao
from test_gpu_attention import BF, F32, Batch, _say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths,earlier,hq,hkv,cut", FORMS)
@pytest.mark.parametrize("D,f32", TYPES)
def test_attention_of_256_rows(D, f32, lengths, earlier, hq, hkv, cut, monkeypatch):
    want = None
    for page in (0, 16, 7):
        _say("attention, 256 rows", D, "f32" if f32 else "bf16", lengths, earlier, "page", page)
        b = Batch(37, lengths, hq, hkv, D, F32 if f32 else BF, earlier=earlier, page=page)
        assert (b.ws_bytes > 0) == cut
        if want is None:      # the same queries, keys and values for all of them
            want = ao.causal_attention(b.q64, b.k64, b.v64, b.cu_host, b.ck_host)
            monkeypatch.setattr(ao, "causal_attention", lambda *a, **k: want)
        b.run()
        b.check()
