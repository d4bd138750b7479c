// The form that a call of seg_attn_paged_chosen or seg_kv_paged_reserve takes, from the library's own rules (linked from libsegattn.so).  One
// call per input line, one answer per output line:
//   reserve heads sequences page_rows n_pages per_head total longest
//       -> "one" (workgroup) | "four" (launches)
//   D Hq Hkv policy S T batch total longest max_rows block_rows n_chosen e4m3 out_fp32
//       -> listed blocks: "blocks" (a block once for the tokens that list it) | "tokens"; tokens of a part;
//          windows: "shares" (cut evenly) | "units" (a workgroup each) | "tokens"; workgroups of the windows;
//          bytes that the form lays out; bytes that the library asks for
// (policy: a digit per KV head.)  Needs no GPU.
#include <iostream>
#include <sstream>
#include <string>
#include <vector>

#include "segattn_paged_api.hip"  // build_paged, build_pages, chosen_space

static bool reserve(const std::string &line) {
  std::istringstream in(line);
  std::string word;
  long long total, longest;
  int page_rows;
  Problem p;
  PagedCache c;
  in >> word >> p.Hkv >> p.B >> page_rows >> c.n_pages >> c.per_head >> total >> longest;
  if (in.fail() || !batch_size_fits(p, total, longest)) return false;
  c.page_rows = fast_div_by(page_rows);
  std::cout << (reserve_by_one_workgroup(p, c, total, longest) ? "one" : "four") << '\n';
  return true;
}

static bool answer(const std::string &line) {
  std::istringstream in(line);
  segattn_config cfg;
  memset(&cfg, 0, sizeof(cfg));
  std::string text;
  long long total, longest, max_rows;
  int block_rows, n_chosen, e4m3;
  in >> cfg.head_dim >> cfg.n_q_heads >> cfg.n_kv_heads >> text >> cfg.seg_len >> cfg.tail_len >> cfg.batch >> total >> longest >> max_rows >> block_rows >>
      n_chosen >> e4m3 >> cfg.out_fp32;
  std::vector<uint8_t> policy;
  for (char x : text) policy.push_back((uint8_t)(x - '0'));
  cfg.kv_policy = policy.data();
  segattn_pages pages;
  memset(&pages, 0, sizeof(pages));
  pages.k = pages.v = (void *)4096;
  pages.k_scale = pages.v_scale = (uint8_t *)4096;
  pages.table = (const int32_t *)4096;
  pages.type = e4m3 ? SEGATTN_PAGES_E4M3 : SEGATTN_PAGES_BF16;
  pages.page_rows = block_rows;
  pages.max_pages = (int32_t)((max_rows + block_rows - 1) / block_rows);
  pages.n_pages = 1;
  segattn_blocks blocks = {block_rows, nullptr, nullptr};
  Problem p;
  PagedCache c;
  PagedChosenArgs a;
  unsigned long long bytes;
  memset(&a, 0, sizeof(a));
  if (in.fail() || (int)policy.size() != cfg.n_kv_heads || !build_paged(&cfg, p) || !build_pages(&pages, p, c) || !batch_size_fits(p, total, longest) ||
      !chosen_space(p, c, &blocks, (const int32_t *)4096, total, longest, max_rows, n_chosen, nullptr, a, bytes))
    return false;
  const unsigned long long laid_out = plan_paged_chosen(a, longest, nullptr);
  std::cout << (a.by_block ? "blocks " : "tokens ") << (a.by_block ? a.part_tokens : 0) << ' '
            << (!a.wide_windows ? "tokens " : a.wide_wgs > 0 ? "shares " : "units ") << (a.wide_windows && a.wide_wgs > 0 ? a.wide_wgs : a.wgs_other) << ' ' << laid_out
            << ' ' << seg_attn_paged_chosen_workspace_bytes(&cfg, &pages, &blocks, total, longest, max_rows, n_chosen) << '\n';
  return true;
}

int main() {
  for (std::string line; std::getline(std::cin, line);)
    if (!(line.rfind("reserve ", 0) == 0 ? reserve(line) : answer(line))) {
      std::cout << "refused: " << line << '\n';
      return 1;
    }
}
