// Runs on the CPU the device code that cuts a sequence's keys into parts (laps_kv4_part_rounds).  Reads lines of
//   kv_len max_pages parts min_parts
// and prints rounds a part and parts.
#define main shares_main
#include "attn_shares_driver.cpp"
#undef main

int main() {
    int kv_len, max_pages, parts, min_parts;
    while (std::scanf("%d %d %d %d", &kv_len, &max_pages, &parts, &min_parts) == 4) {
        int used = -1;
        const int each = laps_kv4_part_rounds(kv_len, max_pages, parts, min_parts, &used);
        std::printf("%d %d\n", each, used);
    }
    return 0;
}
