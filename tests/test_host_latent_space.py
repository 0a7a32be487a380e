"""CPU tests of the workspace of attention to latent caches: one that is sized for the longest step of a program serves its shorter ones."""
import itertools

import pytest

import paper_2403_11805_amd as kvs


def shape(heads, latent=512, n_tokens=3008):
    return kvs.LatentShape(1, heads, latent, 64, 128, 128, n_tokens, 16, 64)


@pytest.mark.parametrize("heads", [1, 2, 4, 5, 8, 9, 12, 16, 24, 32, 40, 42, 43, 48, 64, 65, 96, 100, 128, 129, 130, 192, 193, 1024])
def test_more_rows_or_sequences_never_take_less(heads):
    seqs = (1, 2, 3, 8, 24, 64, 200, 256, 257, 300, 900)
    for latent, n_tokens in itertools.product((256, 512), (16, 3008, 32768)):
        s = shape(heads, latent, n_tokens)
        need = {}
        for n, m in itertools.product(seqs, range(1, 17)):
            if n * m * (heads * (latent // 128) + 1) <= 1 << 20:            # (far more than that is refused)
                need[n, m] = kvs.kv_latent_attend_workspace_bytes(s, n, m)
        assert len(need) >= 16
        for (n, m), mine in need.items():
            for less in ((n, m - 1), (seqs[max(seqs.index(n) - 1, 0)], m)):
                assert need.get(less, 0) <= mine, (latent, n_tokens, n, m, less)


def test_longer_sequences_never_take_less():
    for heads, m in itertools.product((4, 16, 40), (1, 3, 4, 8, 9, 16)):
        need = [kvs.kv_latent_attend_workspace_bytes(shape(heads, 512, n), 3, m) for n in (16, 32, 48, 160, 1008, 3008, 32768)]
        assert need == sorted(need), (heads, m)


def test_more_tokens_of_prompts_never_take_less():
    s = shape(16)
    need = [kvs.kv_latent_prompts_workspace_bytes(s, 7, n) for n in range(1, 500)]
    assert need == sorted(need)
    need = [kvs.kv_latent_prompts_workspace_bytes(s, n, 200) for n in range(1, 500)]
    assert need == sorted(need)
