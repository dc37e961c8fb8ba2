"""Products grouped by expert that are many tiles to every workgroup of the persistent kernel, against 64 bits: what is handed on from one tile to
the next (the streams of slabs, the vectors' two buffers, the row numbers, 1 / S_a) shows from a workgroup's second and third tile on."""
import pytest
import torch

import moe_reference as R
import test_gpu_gemm_grouped as G
from paper_2310_17723_amd import binding as HB

pytestmark = pytest.mark.gpu

DTYPE = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn, "bf16": torch.bfloat16, "f16": torch.float16}
# per form: rows and columns of a tile, workgroups, and N such that the rows below are three tiles and more to every one of them
FORMS = {128: (128, 128, 512, 7301), 256: (256, 256, 256, 13061), 384: (256, 128, 256, 6603)}
COUNTS = [700, 1, 0, 300, 2, 1500, 129, 257]                             # several row tiles of an expert, single rows, none; full tiles and others
BEHIND = 5


def _tiles(tile):
    """The least number of tiles (at the full height; lower ones make more)."""
    bm, bn, _, N = FORMS[tile]
    return sum(-(-n // bm) for n in COUNTS) * -(-N // bn)


class Walk:
    def __init__(self, fmt, tile, K, gathered, row_scale, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.rand(s, device="cuda", generator=g)  # noqa: E731
        self.fmt, self.tile, self.K, self.E, self.N = fmt, tile, K, len(COUNTS), FORMS[tile][3]
        self.R = sum(COUNTS) + BEHIND
        MA = 999 if gathered else self.R
        self.index = torch.randint(0, MA, (self.R,), device="cuda", generator=g).int() if gathered else None
        self.offsets = torch.tensor([sum(COUNTS[:e]) for e in range(self.E + 1)], dtype=torch.int32, device="cuda")

        def codes(*shape):
            if fmt == "i8":
                return torch.randint(-127, 128, shape, device="cuda", generator=g, dtype=torch.int8)
            x = torch.randn(shape, device="cuda", generator=g)
            return (x * 60).clamp(-448, 448).to(DTYPE[fmt]) if fmt == "e4m3" else x.to(DTYPE[fmt])
        self.A, self.W = codes(MA, K), codes(self.E, self.N, K)
        # every column of every expert has a size of its own, from 1/8 to 8: another's vectors, or an older tile's, are far off
        self.size = torch.exp2(torch.randint(-3, 4, (self.E, self.N), device="cuda", generator=g).float())
        one = {"i8": 73.0 * 73.0, "e4m3": 60.0 * 60.0}.get(fmt, 1.0) * K ** 0.5
        self.rs = 0.5 + 1.5 * rand(MA) if row_scale else None
        self.cs = self.size * (0.7 + 0.6 * rand(self.E, self.N)) / one if fmt in ("i8", "e4m3") else None
        if self.cs is None:
            self.W *= (1.0 / K ** 0.5)
            self.W *= self.size[..., None].to(self.W.dtype)              # (powers of two)
        self.bias = self.size * torch.randn((self.E, self.N), device="cuda", generator=g)
        self.os = self.size * (0.01 + 0.04 * rand(self.E, self.N))

    def run(self, hero, epi, out_dt, tile):
        N4 = self.N + -self.N % 4
        whole = torch.full((self.R, N4 * out_dt.itemsize), 91, dtype=torch.uint8, device="cuda")
        out = whole.view(out_dt)[:, :self.N]
        kw = dict(row_index=self.index, bias=self.bias, C_out=out, tile=tile)
        if self.cs is None:
            hero.hero_hp_gemm_grouped(self.A, self.W, self.offsets, gelu=epi == "gelu", **kw)
        else:
            fn = hero.hero_int8_gemm_grouped if self.fmt == "i8" else hero.hero_fp8_gemm_grouped
            cs = self.cs * 30 if epi == "requant" else self.cs
            fn(self.A, self.W, self.offsets, a_row_scale=self.rs, b_col_scale=cs, epi=R.EPI_OF[epi], out_col_scale=self.os if epi == "gelu_requant" else None, **kw)
        assert (whole[sum(COUNTS):] == 91).all() and (whole[:, self.N * out_dt.itemsize:] == 91).all(), "rows and columns that are nobody's"
        return out

    def check(self, got, epi):
        """All rows of all experts.  u = 2^-24.  slack: of the fp32 value in front of the epilogue's last rounding."""
        u, at = 2.0 ** -24, 0
        for e, n in enumerate(COUNTS):
            if n == 0:
                continue
            src = slice(at, at + n) if self.index is None else self.index[at:at + n].long()
            a = (self.A.view(torch.uint8)[src].view(self.A.dtype) if self.A.element_size() == 1 else self.A[src]).double()
            w, bias = self.W[e].double(), self.bias[e].double()
            s = torch.ones((), dtype=torch.float64, device="cuda")
            if self.cs is not None:
                s = (self.cs[e] * 30 if epi == "requant" else self.cs[e]).double()
                if self.rs is not None:
                    s = s * self.rs[src].double()[:, None]
            t = (a @ w.t()) * s
            y = t + bias
            if self.fmt == "i8":                                          # the sum is exact, its conversion and the row scale round: 2 u of t
                slack = 2 * u * t.abs()
            else:
                # the sum of K products in fp32, K u of sum |a w|; E4M3: groups of eight with 13 fractional bits below the largest, 2^-10 of it more
                slack = (self.K * u + (2.0 ** -10 if self.fmt == "e4m3" else 0.0)) * (a.abs() @ w.abs().t()) * s + 2 * u * t.abs()
            slack = (slack + u * y.abs()) * (1 + 2.0 ** -20)              # the fused (or plain) addition of the bias; products of these errors
            if epi in ("gelu", "gelu_requant"):                           # |GELU'| < 1.13; its fp32 form is off by 2^-23 and the last step's u
                slack = 1.13 * slack + 2.0 ** -23
                y = R.gelu(y)
                slack = slack + u * y.abs()
            if epi == "gelu_requant":                                     # 1 / S_a (E4M3: to one step) and the product with it
                y, slack = y / self.os[e].double(), slack / self.os[e].double()
                slack = (slack + 4 * u * y.abs()) * (1 + 2.0 ** -20)
            x = got[at:at + n].float().double()
            if got.dtype is torch.int8:
                y, bound = y.clamp(-127, 127), 0.5 + slack
            else:
                half, tiny = {torch.float8_e4m3fn: (2.0 ** -4, 2.0 ** -10), torch.float16: (2.0 ** -11, 2.0 ** -25), torch.bfloat16: (2.0 ** -8, 0.0)}[got.dtype]
                y = y.clamp(-448, 448) if got.dtype is torch.float8_e4m3fn else y
                bound = slack + half * (y.abs() + slack) + tiny
            d = (x - y).abs()
            assert bool((d <= bound).all()), (epi, e, float((d / bound).max()), (d > bound).nonzero()[:4].tolist())
            at += n


@pytest.mark.parametrize("gathered", [False, True], ids=["in_order", "gathered"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3", "bf16", "f16"])
@pytest.mark.parametrize("tile", [128, 256, 384])
def test_three_tiles_and_more_to_a_workgroup(hero, tile, fmt, gathered):
    """The shortest K that the kernel takes (512 bytes), an odd number of pairs of slabs, and a longer one."""
    assert _tiles(tile) >= 3 * FORMS[tile][2] + 56                       # (so that the least that an XCD gets, an eighth less 7, is three to a workgroup)
    size = DTYPE[fmt].itemsize
    for i, k_bytes in enumerate((512, 640, 1664)):
        p = Walk(fmt, tile, k_bytes // size, gathered, size == 1 and (gathered or i != 1), seed=10 * tile + i)
        wide = DTYPE[fmt] if size == 2 else (torch.bfloat16, torch.float16)[i % 2]
        for epi, out_dt in (("dequant", wide), ("gelu", wide), ("requant", DTYPE[fmt]), ("gelu_requant", DTYPE[fmt])):
            if size == 2 and epi not in ("dequant", "gelu"):
                continue
            got = p.run(hero, epi, out_dt, tile)
            p.check(got, epi)
            bits = lambda x: x.view(torch.uint8 if x.dtype.itemsize == 1 else torch.int16)  # noqa: E731
            assert torch.equal(bits(p.run(hero, epi, out_dt, tile)), bits(got)), "the same call again"
            if fmt == "i8":                                               # (to the bit what the kernel of every size gives)
                assert torch.equal(bits(p.run(hero, epi, out_dt, 1)), bits(got))


def test_weights_and_results_beyond_4_gb_in_tiles_of_256_by_128(hero):
    G.test_weights_and_results_beyond_4_gb(hero, 384)


@pytest.mark.parametrize("fmt", ["i8", "e4m3", "bf16"])
def test_the_longest_rows(hero, fmt):
    """K of 2^31 - 64 bytes: a number of bytes, a little more of which 32 bits do not hold."""
    K, dt = (2 ** 31 - 64) // DTYPE[fmt].itemsize, DTYPE[fmt]
    A, W = (torch.zeros(K, dtype=torch.uint8 if dt.itemsize == 1 else dt, device="cuda").view(dt) for _ in range(2))
    at = [0, 1, K // 3, K // 2, K - 33, K - 2, K - 1]
    for i, k in enumerate(at):                                            # (single elements, through the type's own conversion)
        A[k:k + 1] = torch.tensor([i + 1.0]).to(dt).cuda()
        W[k:k + 1] = torch.tensor([2.0]).to(dt).cuda()
    off, want = torch.tensor([0, 1], dtype=torch.int32, device="cuda"), 2.0 * sum(range(1, len(at) + 1))
    for tile in (None, 1):
        out = torch.zeros((1, 4), dtype=torch.bfloat16, device="cuda")
        kw = dict(C_out=out[:, :1], tile=tile)
        if fmt == "bf16":
            hero.hero_hp_gemm_grouped(A[None], W[None, None], off, **kw)
        else:
            fn = hero.hero_int8_gemm_grouped if fmt == "i8" else hero.hero_fp8_gemm_grouped
            fn(A[None], W[None, None], off, b_col_scale=torch.ones((1, 1), device="cuda"), **kw)
        assert out[0].tolist() == [want, 0, 0, 0]


@pytest.mark.parametrize("tile", G.TILES)
def test_rows_gathered_from_between_2_and_4_gb(hero, tile):
    """Byte offsets of 32 bits, the uppermost of which is set: they are no negative numbers.  (As much memory of the test's own lies in front of the rows.)"""
    MA, K, N = 2 ** 20 - 3, 4096, 48
    room = torch.zeros((2 ** 19 + MA, K), dtype=torch.int8, device="cuda")
    room[:2 ** 19] = 1
    A = room[2 ** 19:]
    index = torch.tensor([0, MA - 1, 2 ** 19, 2 ** 19 - 1, 700_001, MA - 2, 77], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(7)
    A[index.long()] = torch.randint(-127, 128, (7, K), generator=g, device="cuda", dtype=torch.int8)
    W = torch.randint(-127, 128, (2, N, K), generator=g, device="cuda", dtype=torch.int8)
    rs = torch.ones(MA, device="cuda")
    rs[index.long()] = torch.arange(1.0, 8.0, device="cuda")
    off, cs = torch.tensor([0, 3, 7], dtype=torch.int32, device="cuda"), torch.full((2, N), 1e-4, device="cuda")
    got = hero.hero_int8_gemm_grouped(A, W, off, row_index=index, a_row_scale=rs, b_col_scale=cs, tile=tile).double()
    for e, (a, b) in enumerate(((0, 3), (3, 7))):
        y = A[index[a:b].long()].double() @ W[e].double().t() * rs[index[a:b].long()].double()[:, None] * cs[e].double()
        assert bool(((got[a:b] - y).abs() <= (2.0 ** -8 + 2.0 ** -20) * y.abs()).all())      # one rounding to BF16, a few of fp32
