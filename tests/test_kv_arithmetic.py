"""Arithmetic of the attention's schedule and addresses at its ends (CPU)."""
import host_code


def test_shares_of_a_kernel_that_is_not_launched(tmp_path):
    """Behind shared prefixes a row's sources are looked up by the cuts of both kernels: the one that is
    not launched has no requests, and asking for their shares is defined."""
    out = host_code.run(tmp_path, "kv_sched.h", r'''
    int32_t start[] = {0, 5}, first[] = {0, 1}, context[] = {40};
    KvSharedArgs a{};
    a.R = 1;
    a.T = 5;
    a.groups = 1;
    a.G = 2;
    a.shift = 4;
    a.W = a.p_W = 4;
    a.start = a.p_start = start;
    a.first = first;
    a.context = a.p_context = context;
    KvCut none{}, many{};
    many.rows = 8;
    for (const KvCut &c : {none, many})
        for (int r = 0; r < 2; ++r) {
            const KvShare s = kv_share(a, c, r);
            std::printf("%d %d ", s.n, s.ctx);
            if (c.rows == 8) std::printf("%d ", s.tiles);
        }
''')
    assert out.split() == "5 40 5 40 5 40 2 5 40 2".split()


def test_rows_of_codes_far_apart(tmp_path):
    """The last row of 16 in the widest strides that the entry points take: blocks of 16 tokens end
    below 2^31 bytes."""
    out = host_code.run(tmp_path, "kv_types.h", r'''
    const int64_t four = (1ll << 28) - 32, eight = (1ll << 27) - 32, sixteen = (1ll << 26) - 8;
    std::printf("%u %u ", row_bytes<mx4>(15, four, 255), row_bytes<mx4>(12, four, 0));
    std::printf("%u %u %u ", row_bytes<mx8>(15, eight, 255), row_bytes<fp8>(15, eight, 7), row_bytes<bf16>(15, sixteen, 9));
    std::printf("%u ", row_bytes<mx4>(15, 0, 31));
''')
    four, eight, sixteen = (1 << 28) - 32, (1 << 27) - 32, (1 << 26) - 8
    assert [int(x) for x in out.split()] == [(15 * four + 255) // 2, 6 * four, 15 * eight + 255, 15 * eight + 7,
                                             2 * (15 * sixteen + 9), 15]
    assert 16 * four // 2 < 2 ** 31
