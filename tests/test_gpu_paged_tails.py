"""Attention over pages where the output is the softmax's tail (run with -m gpu): one key far above the others, with a value of zero, and thousands of
keys below it, whose probabilities are small as 16-bit numbers.  Every form of the kernels against 64 bits."""
import pytest
import torch

from tests.paged_helpers import attend64, attention_bound, ints, offsets, random_cache

pytestmark = pytest.mark.gpu

# Beside what attention_bound allows (u of each probability, or 2^-15 where it goes in as two terms): what lies below fp16's normal numbers is off by an
# absolute 2^-25, where the largest probability is 2^9 (chunks) or 2^12 (few queries, here with a factor of two).
ABSOLUTE = {True: 2.0 ** -36, False: 2.0 ** -34}                 # of the largest probability; True: two terms
MOST = 5.0                                                       # bound on the values

# new tokens, cached ones, heads per kv head, kv heads, head size, bound on the length that the call names (0: its own), two terms
FORMS = {"one": ([1] * 3, [2500, 100, 1700], 1, 200, 64, 0, True), "spans": ([1, 1], [4000, 300], 4, 2, 128, 0, True),
         "few": ([4, 3], [4000, 3000], 4, 2, 64, 0, True), "sixteens": ([5, 9, 2], [900, 300, 600], 4, 8, 128, 0, True),
         "ranges": ([40, 65], [4000, 900], 4, 2, 128, 60000, False), "tiles": ([40, 65, 50] * 4, [500, 900, 20] * 4, 4, 8, 64, 400, False),
         "groups": ([64] * 16, [1000] * 16, 4, 8, 64, 0, False), "wide": ([1400, 1300], [2000, 900], 16, 8, 128, 0, False)}


@pytest.fixture(scope="module")
def qt():
    import paper_2602_10431_amd as pkg
    pkg.load_library()
    return pkg


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("near,far", [(12.0, 16.0), (15.0, 15.0), (18.0, 22.0)])
@pytest.mark.parametrize("form", sorted(FORMS))
def test_one_key_far_above_the_others(qt, form, near, far, dtype):
    new, old, rep, nkv, d, bound, split = FORMS[form]
    lens, page, scale = [o + n for o, n in zip(old, new)], 64, 0.125
    if bound and bound < max(lens):                              # the call's bound cuts the sequences
        old = [min(o, bound - n) for o, n in zip(old, new)]
        lens = [o + n for o, n in zip(old, new)]
    kv, slots = random_cache(qt, lens, page, nkv, d, dtype, 3)
    g = torch.Generator(device="cuda").manual_seed(7)
    # queries of ones in 64 columns, keys of one number in them: scores are 8 times that number, 20 at the first key (products add up to 160)
    q = torch.zeros(sum(new), rep * nkv, d, dtype=dtype, device="cuda")
    q[..., :64] = 1.0
    below = near + (far - near) * torch.rand(kv.k.shape[0], nkv, page, 1, generator=g, device="cuda")
    kv.k.zero_()
    kv.k[..., :64] = (2.5 - below / 8.0).to(dtype)
    kv.v.copy_(torch.randn(kv.v.shape, generator=g, device="cuda").clamp(-MOST, MOST))
    for s in slots:
        p = int(kv.table[0, s, 0])
        kv.k[p, :, 0, :64], kv.v[p, :, 0] = 2.5, 0.0
    got = qt.qtale_paged_attention(kv, 0, q, offsets(new), first=ints(old), slots=ints(slots), scale=scale, max_new=max(new), max_len=bound or max(lens))
    want, size = attend64(kv, 0, q, new, old, slots, 0, 0, scale)
    keys = torch.repeat_interleave(torch.tensor(lens, device="cuda").double(), torch.tensor(new, device="cuda"))[:, None, None]
    limit = attention_bound(want, size, dtype, split)
    if dtype is torch.float16:
        limit += ABSOLUTE[split] * MOST * keys
    off = (got.double() - want).abs() / limit
    assert float(size.min()) > 0.0 and float(off.max()) <= 1.0, (int((off > 1.0).sum()), float(off.max()))
