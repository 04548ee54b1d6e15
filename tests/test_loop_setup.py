"""What the decoding loop's verifiers set up (CPU: no kernel is launched)."""
import torch

from paper_2608_13076_gb300 import speculative as S


def test_int4_verifier_holds_no_bf16_cache(monkeypatch):
    """A cache in 4 bits is set up at sizes whose bf16 cache would not fit: none is made on the way."""
    made = []

    def spy(name):
        real = getattr(torch, name)

        def f(*args, **kwargs):
            t = real(*args, **kwargs)
            made.append(t)
            return t
        monkeypatch.setattr(torch, name, f)

    for name in ("zeros", "zeros_like", "empty", "empty_like", "full"):
        spy(name)
    cfg, B, cap = S.ToyConfig(), 3, 1000
    v = S.ToyVerifierInt4(cfg, B, cap, seed=1, device="cpu", page=128)
    numbers = B * cfg.Hkv * cap * cfg.D
    assert not [t.shape for t in made if t.dtype == torch.bfloat16 and t.numel() >= numbers]
    assert not hasattr(v, "k_cache") and not hasattr(v, "v_cache")
    codes, params = v.pools[:2]
    assert codes.shape == (24, cfg.Hkv, 128, cfg.D // 2) and params.shape == (24, cfg.Hkv, 128, 1, 2)
    assert v.table.shape == (B, 8) and sorted(v.table.flatten().tolist()) == list(range(24))
    assert v.rope.shape == (1024, cfg.D // 2, 2)


def test_bf16_verifier():
    cfg = S.ToyConfig()
    v = S.ToyVerifier(cfg, 2, 100, seed=1, device="cpu")
    assert v.k_cache.shape == v.v_cache.shape == (2, cfg.Hkv, 100, cfg.D) and v.k_cache.dtype == torch.bfloat16
