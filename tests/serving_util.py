"""A served decoding step's inputs (numpy, seeded) and its calls on the GPU."""
import numpy as np

from oracle import serving as sv
from paper_2505_19342_amd import binding as B
from paper_2505_19342_amd import workloads as wl


class Step:
    """Sequences with `lens` cached and `new` new tokens; pages that hold nothing yet are full of NaN codes and their scales NaN."""

    def __init__(self, dtype, hq, hkv, dh, page, lens, new, seed=0, behind=0, spread=(-8, -5), std=1.3, columns=0):
        rng = self.rng = np.random.default_rng(seed)
        self.dtype, self.hq, self.hkv, self.dh, self.page = dtype, hq, hkv, dh, page
        self.rnd = wl.round_to_bf16 if dtype == "bf16" else (lambda a: np.asarray(a, np.float32))
        held = [-(-(a + b) // page) for a, b in zip(lens, new)]
        self.n_pages = sum(held) + 2
        self.table = np.full((len(lens), max(held + [1, columns - 1]) + 1), -1, np.int32)
        ids = iter(rng.permutation(self.n_pages))
        for s, h in enumerate(held):
            self.table[s, :h] = [next(ids) for _ in range(h)]
        self.lens, self.first = np.array(lens, np.int32), np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        self.n = int(self.first[-1]) + behind
        self.q, self.k, self.v = (self.rnd((rng.standard_normal((self.n, h, dh)) * std).astype(np.float32)) for h in (hq, hkv, hkv))
        shape = (self.n_pages, hkv, page, dh)
        self.pages = [np.full(shape, 127, np.uint8) for _ in range(2)]
        self.scales = [np.full(shape[:2], np.nan, np.float32) for _ in range(2)]
        for s, h in enumerate(held):
            for i in range(h):
                here = min(max(lens[s] - i * page, 0), page)             # tokens of the page that are cached
                if here:
                    for j in range(2):
                        self.pages[j][self.table[s, i], :, :here] = sv.e4m3_code(np.clip(rng.standard_normal((hkv, here, dh)) * 83, -448, 448))
                        self.scales[j][self.table[s, i]] = 2.0 ** rng.integers(*spread, hkv)

    def fill(self):
        """Every token of the step cached, the new ones' codes made up."""
        for s in range(len(self.lens)):
            for i in range(self.first[s + 1] - self.first[s]):
                t = self.lens[s] + i
                p = self.table[s, t // self.page]
                for j in range(2):
                    self.pages[j][p, :, t % self.page] = sv.e4m3_code(np.clip(self.rng.standard_normal((self.hkv, self.dh)) * 83, -448, 448))
                    self.scales[j][p] = np.where(np.isnan(self.scales[j][p]), np.float32(2.0 ** -6), self.scales[j][p])
        return self

    def desc(self, **more):
        return B.cache_desc(self.dtype, self.hq, self.hkv, self.dh, self.page, self.n_pages, len(self.lens), self.table.shape[1], self.n, **more)


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


def attend(st, prior=None, prior_lse=None, scale=0.0, want_lse=True, **more):
    import torch
    from gpu_util import empty_like_dtype, to_dev, to_host
    d = st.desc(scale=scale, **more)
    out = empty_like_dtype((st.n, st.hq, st.dh), st.dtype).fill_(7.0)
    lse = torch.full((st.n, st.hq), 7.0, device="cuda:0") if want_lse else None
    ws = torch.full((B.astra_cache_attention_workspace_bytes(d),), 255, dtype=torch.uint8, device="cuda:0")          # NaN everywhere
    B.astra_cache_attention(d, dev(st.table), dev(st.lens), dev(st.first), to_dev(st.q, st.dtype), dev(st.pages[0]), dev(st.pages[1]), dev(st.scales[0]),
                            dev(st.scales[1]), None if prior is None else to_dev(prior, st.dtype), None if prior is None else dev(prior_lse), out, lse, ws)
    torch.cuda.synchronize()
    return to_host(out), None if lse is None else lse.cpu().numpy()


def attention_bar(st, ref, scale):
    """How far out may be from the 64-bit result, by its arithmetic (u = 2^-24): a score is a sum of dh products in at most dh / 32 * 3 + 32 roundings and two
    more for its scale, taken off a reference and exponentiated (1 ulp): |ds| <= (dh / 8 + 40) u S for S = max sum |q k| scale.  Both a weight and
    the sum of weights carry that; the sum over T values in fp32 adds (T / 32 + 64) u, two bf16 parts of a weight 2^-16 (three: nothing); all relative
    to the largest |value|.  The rounding of the result is half a step."""
    val = sv.e4m3_values()
    kmax, vmax = ((np.abs(np.nan_to_num(val[p])).max() * np.nanmax(s, initial=0.0)) for p, s in zip(st.pages, st.scales))
    u = 2.0 ** -24
    f = scale or st.dh ** -0.5
    s = min(np.abs(st.q).sum(2).max() * kmax, np.linalg.norm(st.q, axis=2).max() * kmax * st.dh ** 0.5) * f
    total = float((st.lens + np.diff(st.first)).max(initial=1))
    rel = 2 * (st.dh / 8 + 40) * u * s + (total / 32 + 64) * u + (2.0 ** -16 if st.dtype == "bf16" else 0.0)
    return rel * vmax + (2.0 ** -8 if st.dtype == "bf16" else 2.0 ** -24) * np.abs(ref), (st.dh / 8 + 40) * u * s + (total / 32 + 64) * u


def check_attention(st, prior=None, prior_lse=None, scale=0.0, **more):
    ref, ref_lse = sv.cache_attention(st.table, st.lens, st.first, st.q, st.pages[0], st.pages[1], st.scales[0], st.scales[1], scale or None, prior, prior_lse)
    out, lse = attend(st, prior, prior_lse, scale, **more)
    n = st.first[-1]
    bar, bar_lse = attention_bar(st, ref[:n], scale)
    if prior is not None:
        bar = bar + 2.0 ** -20 * np.abs(np.nan_to_num(prior[:n]))
    off, off_lse = np.abs(out[:n] - ref[:n]), lse[:n] - ref_lse[:n]
    print(f"max off {off.max(initial=0):.2e} of {np.min(bar, initial=np.inf):.2e}, lse {np.nanmax(np.abs(off_lse), initial=0):.2e} of {bar_lse:.2e}")
    assert np.all(off <= bar)
    none = np.isneginf(ref_lse[:n])
    assert np.array_equal(none, np.isneginf(lse[:n])) and np.all(out[:n][none] == 0)
    assert np.all(np.abs(off_lse[~none]) <= bar_lse + 2.0 ** -22 * np.abs(ref_lse[:n][~none]))
    assert np.all(out[n:] == 7.0) and np.all(lse[n:] == 7.0)                       # rows behind the last sequence
    return out, lse
