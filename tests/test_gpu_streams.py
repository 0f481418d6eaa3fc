"""Calls on streams of the caller's: memory that a call takes for its results and its staging must not be memory
that the current stream's pending work still uses."""
import numpy as np
import pytest
import torch

import paper_2410_15240_amd as F

pytestmark = pytest.mark.gpu

KEY, IV, CHAIN, SIZE, CHUNK = bytes(range(32)), bytes(range(100, 112)), 4096, 300_000, 1 << 16


@pytest.fixture(scope="module")
def calls():
    gen = torch.Generator(device="cuda").manual_seed(5)
    pt = torch.randint(0, 256, (SIZE,), dtype=torch.uint8, device="cuda", generator=gen)
    ct, tags = F.encrypt_tag(KEY, IV, CHAIN, pt)
    ks = F.keystream(KEY, IV, CHAIN, SIZE)
    h_ct, h_tags = ct.cpu().pin_memory(), tags.cpu()
    off = np.arange(0, SIZE, CHAIN, dtype=np.uint64)
    ln = np.minimum(CHAIN, SIZE - off)
    one = lambda fn, *a: lambda s: fn(*a, **({} if s is None else dict(stream=s[0])))

    def eager(s):
        r = F.decrypt_eager(KEY, IV, CHAIN, ct, tags, **({} if s is None else dict(decrypt_stream=s[0], verify_stream=s[1])))
        return r.plaintext, r.ok

    def h2d(**kw):
        return lambda s: F.pipeline_h2d(KEY, IV, CHAIN, h_ct, h_tags, chunk_bytes=CHUNK, **kw,
                                        **({} if s is None else dict(copy_stream=s[0], compute_stream=s[1], verify_stream=s[2])))

    def d2h(**kw):
        return lambda s: F.pipeline_d2h(KEY, IV, CHAIN, pt, chunk_bytes=CHUNK, **kw,
                                        **({} if s is None else dict(copy_stream=s[0], compute_stream=s[1])))

    return {
        "encrypt": one(F.encrypt_tag, KEY, IV, CHAIN, pt), "decrypt": one(F.decrypt_verify, KEY, IV, CHAIN, ct, tags),
        "keystream": one(F.keystream, KEY, IV, CHAIN, SIZE), "apply": one(F.apply_verify, KEY, IV, CHAIN, ct, ks, tags),
        "encrypt-ragged": one(F.encrypt_tag_ragged, KEY, IV, off, ln, pt),
        "decrypt-ragged": one(F.decrypt_verify_ragged, KEY, IV, off, ln, ct, tags), "eager": eager,
        "h2d": h2d(depth=0), "h2d-ring": h2d(depth=2), "h2d-eager": h2d(depth=3, mode=F.PIPE_EAGER),
        "h2d-otp": h2d(depth=2, mode=F.PIPE_OTP), "h2d-direct": h2d(mode=F.PIPE_DIRECT),
        "d2h": d2h(), "d2h-direct": d2h(mode=F.PIPE_DIRECT),
    }


@pytest.mark.parametrize("name", ["encrypt", "decrypt", "keystream", "apply", "encrypt-ragged", "decrypt-ragged", "eager", "h2d",
                                  "h2d-ring", "h2d-eager", "h2d-otp", "h2d-direct", "d2h", "d2h-direct"])
def test_memory_that_the_current_stream_still_reads_is_left_alone(calls, name, monkeypatch):
    call, sides = calls[name], [torch.cuda.Stream() for _ in range(3)]
    made, empty = [], torch.empty

    def counting(*a, **kw):
        t = empty(*a, **kw)
        if t.is_cuda:
            made.append((t.data_ptr(), t.numel()))
        return t

    with monkeypatch.context() as m:
        m.setattr(torch, "empty", counting)
        results = call(None)
    torch.cuda.synchronize()
    want = [t.cpu().clone() for t in (results if isinstance(results, tuple) else (results,))]
    sizes = [n for _, n in made]
    del results
    for s in sides:     # (the key's tables, on every stream)
        F.keystream(KEY, IV, CHAIN, 64, stream=s)
    torch.cuda.synchronize()
    freed = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
    places = {t.data_ptr() for t in freed}
    torch.cuda._sleep(100_000_000)
    copies = [t.clone() for t in freed]     # queued behind the wait, reading memory that is free for this stream's next calls
    del freed
    made.clear()
    with monkeypatch.context() as m:
        m.setattr(torch, "empty", counting)
        results = call(sides)
    assert len(made) == len(sizes) and not places & {p for p, _ in made}
    for s in sides:
        s.synchronize()
    for got, t in zip(results if isinstance(results, tuple) else (results,), want):
        assert torch.equal(got.cpu(), t)
    assert all(bool((c == 7).all()) for c in copies)
