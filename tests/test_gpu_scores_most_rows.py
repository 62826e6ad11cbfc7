"""Log probabilities of more rows than one launch has threads for (2^32 in a direction of its grid)."""
import pytest

torch = pytest.importorskip("torch")
import paper_2306_03078_amd.block_binding as K  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


def test_log_probabilities_of_two_to_the_24_rows():
    """Two logits a row: log probabilities and entropies go by their difference d, and are those of a row on its own."""
    rows = (1 << 24) + 5
    d = (torch.arange(rows, device="cuda") % 11).half()
    logits = torch.stack([torch.zeros_like(d), d], 1)
    s = K.SpQRScores(rows, 2, given=1, top=1)
    for t in (s.logprob, s.entropy, s.top_token, s.top_logprob):
        t.fill_(7)
    tokens = torch.arange(rows, dtype=torch.int32, device="cuda")[:, None] % 2
    K.spqr_token_logprobs(s, logits, tokens)
    few = K.SpQRScores(22, 2, given=1, top=1)
    K.spqr_token_logprobs(few, logits[:22], tokens[:22].contiguous())
    at = torch.arange(rows, device="cuda") % 22          # 11 differences, 2 tokens
    for a, b in ((s.logprob, few.logprob), (s.entropy, few.entropy), (s.top_token, few.top_token), (s.top_logprob, few.top_logprob)):
        assert torch.equal(a, b[at])
