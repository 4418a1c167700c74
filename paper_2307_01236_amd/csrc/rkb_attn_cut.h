// Which form of attention's forward takes a call.  Plain C++, so that tests ask it on the host.
#pragma once
#include <cstdint>

namespace rkb {

// k_attn_few takes 32 rows (queries of the heads that share a key head) in a pass over the keys, k_attn 128 queries of one head.  Up to 32
// queries, however many heads share their keys, the first makes no more passes than the second: ceil(queries group / 32) and group.  Its
// pass costs about as much (less over a cache, where k_attn converts the codes again in every pass, more with a bias, which it looks up by bucket); for heads
// of up to 64 columns without a bias it costs half.  16 sequences of 4096 tokens, 4 key heads, bf16, us few / many:
//   columns                  group       1 query    8        16        32        40        64
//   128                          1         34/29    35/30    35/30     35/31     38/32     39/34
//   128                          4         35/68    35/67    38/67     54/68     84/71     89/75
//   128                         16        35/220   54/225   84/232   165/232   207/240   329/249
//   128, over a cache            1         29/34    30/33    30/34     31/35     33/35     33/37
//   128, over a cache            4         29/92    31/94    33/93     51/93     80/97     82/97
//   128, over a cache           16        30/329   51/330   82/328   157/331   192/332   297/334
//   128, a bias                  4         42/70    43/70    49/70     71/72    102/75    107/78
//   256                          4        60/148   64/156   91/159   152/163   265/171   270/174
//   256, over a cache            4        42/218   45/219   65/220   109/222   190/226   192/229
//   64                           1         19/21    19/21    19/21     19/21     19/21     19/22
//   64                           4         19/49    19/50    19/51     27/50     35/51     37/54
//   64, over a cache            16        16/211   32/217   50/217    87/217   105/219   160/220
//   64, a bias                   4         27/52    28/53    33/53     47/54     72/56     72/57
// The rule is the same for tensors and for a cache, so that attention over a cache gives the bits that it gives over the values the cache stands
// for.  Over a cache, wider heads without a bias would still be faster by the first form: 1.1 to 1.7 times at 40
// queries, 1.1 to 1.2 at 64.
inline bool few_queries_win(int64_t queries, int64_t columns, bool bias) { return queries <= (columns <= 64 && !bias ? 64 : 32); }

}  // namespace rkb
